// Reading elements that start anywhere in a 16-byte granule of memory: whole granules, cut.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

namespace liec {

// The 16 bytes from byte `shift` on (below 16, a multiple of the element's size) of two granules.
template <int ELEMENT>
__device__ __forceinline__ uint4 cut_granules(uint4 a, uint4 b, uint32_t shift) {
    const bool two = (shift & 8u) != 0, one = (shift & 4u) != 0;
    const uint32_t v0 = two ? a.z : a.x, v1 = two ? a.w : a.y, v2 = two ? b.x : a.z, v3 = two ? b.y : a.w, v4 = two ? b.z : b.x;
    const uint32_t w0 = one ? v1 : v0, w1 = one ? v2 : v1, w2 = one ? v3 : v2, w3 = one ? v4 : v3;
    if constexpr (ELEMENT >= 4) {
        return make_uint4(w0, w1, w2, w3);
    } else {
        const uint32_t w4 = one ? (two ? b.w : b.y) : v4, half = (shift & 2u) * 8u;
        return make_uint4(__funnelshift_r(w0, w1, half), __funnelshift_r(w1, w2, half), __funnelshift_r(w2, w3, half), __funnelshift_r(w3, w4, half));
    }
}

}  // namespace liec
