// Arrays of up to three axes in front of their columns: whether one overlaps itself or another.
#pragma once
#include <initializer_list>
#include <utility>

#include "overlap.h"

namespace liec {

struct Axes {
    int64_t n[3], s[3];   // entries and steps in bytes, inner first
    int used = 0;
    int64_t base, width;  // bytes of one run of columns
    int64_t end() const {
        int64_t e = base + width;
        for (int i = 0; i < used; ++i) e += (n[i] - 1) * s[i];
        return e;
    }
};

// n, s: outer to inner, all n >= 1, steps in elements >= 0.  Axes of one entry or without a step fall away, axes that
// follow one another without a gap become one.
inline Axes axes_of(const void *base, int64_t cols, int size, std::initializer_list<int64_t> n, std::initializer_list<int64_t> s) {
    Axes a;
    a.base = (int64_t) reinterpret_cast<uintptr_t>(base);
    a.width = cols * size;
    for (int i = (int)n.size() - 1; i >= 0; --i) {
        const int64_t count = n.begin()[i], step = s.begin()[i] * size;
        if (count == 1 || step == 0) continue;
        if (a.used == 0 && step == a.width) a.width *= count;
        else if (a.used > 0 && step == a.n[a.used - 1] * a.s[a.used - 1]) a.n[a.used - 1] *= count;
        else { a.n[a.used] = count; a.s[a.used++] = step; }
    }
    return a;
}

// The runs of an array that is written share no memory: in the order of their steps, every axis steps over all that
// lies within it.
inline bool disjoint(int64_t cols, std::initializer_list<int64_t> n, std::initializer_list<int64_t> s) {
    int64_t count[3], step[3], reach = cols;
    int used = 0;
    for (int i = (int)n.size() - 1; i >= 0; --i)
        if (n.begin()[i] > 1) { count[used] = n.begin()[i]; step[used++] = s.begin()[i]; }
    for (int k = 0; k < used; ++k) {
        int least = k;
        for (int i = k + 1; i < used; ++i)
            if (step[i] < step[least]) least = i;
        std::swap(count[k], count[least]);
        std::swap(step[k], step[least]);
        if (step[k] < reach) return false;
        reach += (count[k] - 1) * step[k];
    }
    return true;
}

// True where a and b share a byte: as `overlap` for up to two axes; a third is walked, up to 1024 pairs of steps
// (beyond them arrays whose ranges cross are taken to be apart).
inline bool meet(const Axes &a, const Axes &b) {
    if (a.end() <= b.base || b.end() <= a.base) return false;
    auto rows = [](const Axes &x, int64_t i) {
        return Rows{x.base + (x.used > 2 ? i * x.s[2] : 0), x.used > 0 ? x.n[0] : 1, x.used > 1 ? x.n[1] : 1, x.used > 0 ? x.s[0] : 0,
                    x.used > 1 ? x.s[1] : 0, x.width};
    };
    const int64_t na = a.used > 2 ? a.n[2] : 1, nb = b.used > 2 ? b.n[2] : 1;
    if (na * nb > 1024) return false;
    for (int64_t i = 0; i < na; ++i)
        for (int64_t j = 0; j < nb; ++j) {
            const Rows x = rows(a, i), y = rows(b, j);
            // (of unequal counts `overlap` can tell blocks only)
            if ((x.rows == y.rows && x.groups == y.groups) || x.block() || y.block()) {
                if (overlap(x, y)) return true;
            }
        }
    return false;
}

}  // namespace liec
