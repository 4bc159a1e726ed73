// The top of a balanced summation tree, joined by one thread.
#pragma once

#ifdef __CUDACC__
#define LIEC_BOTH_SIDES __host__ __device__
#else
#define LIEC_BOTH_SIDES
#endif

namespace liec {

// Balanced binary tree over n >= 1 values, padded to a power of two with zeros, in place.  The zeros are not
// stored: x + 0 is x (for every x but -0, which no sum of squares is), so a value without a partner moves up
// as it is, and nothing beyond s[n - 1] is touched.
LIEC_BOTH_SIDES inline double balanced_join(double *s, int n) {
    while (n > 1) {
        const int pairs = n / 2;
        for (int k = 0; k < pairs; ++k) s[k] = s[2 * k] + s[2 * k + 1];
        if (n & 1) s[pairs] = s[n - 1];
        n = pairs + (n & 1);
    }
    return s[0];
}

}  // namespace liec
