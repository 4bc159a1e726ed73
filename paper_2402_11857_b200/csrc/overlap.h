// Whether two strided arrays share memory: what an entry point can say of its arguments before it launches.
#pragma once
#include <algorithm>
#include <cstdint>

namespace liec {

// groups x rows intervals of `width` bytes; strides in bytes, >= 0.
struct Rows {
    int64_t base, rows, groups, row, group, width;
    int64_t end() const { return base + (rows - 1) * row + (groups - 1) * group + width; }
    bool block() const {   // one interval without gaps
        return (rows == 1 || row == 0 || row == width) && (groups == 1 || group == 0 || group == (rows == 1 || row == 0 ? width : rows * row));
    }
};

inline Rows rows_of(const void *base, int64_t rows, int64_t groups, int64_t row, int64_t group, int64_t cols, int64_t element) {
    Rows r{(int64_t) reinterpret_cast<uintptr_t>(base), rows, groups, row * element, group * element, cols * element};
    if (r.rows == 1) r.row = 0;
    if (r.groups == 1) r.group = 0;
    if (r.rows == 1 || r.row == 0) {   // one axis: the rows
        r.rows = r.groups;
        r.row = r.group;
        r.groups = 1;
        r.group = 0;
    }
    if (r.row == 0) r.rows = 1;
    if (r.group == 0) r.groups = 1;
    return r;
}

inline int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b != 0 && (a < 0) != (b < 0)); }

// Some k in [-limit, limit] with lo < k step < hi (step > 0, or limit = 0).
inline bool multiple_between(int64_t lo, int64_t hi, int64_t step, int64_t limit) {
    if (limit == 0) return lo < 0 && 0 < hi;
    const int64_t first = std::max(-limit, floor_div(lo, step) + 1), last = std::min(limit, -floor_div(-hi, step) - 1);
    return first <= last;
}

// Some interval of a meets [lo, hi).
inline bool meets(const Rows &a, int64_t lo, int64_t hi) {
    for (int64_t g = 0; g < a.groups; ++g) {
        const int64_t at = a.base + g * a.group;   // row i is [at + i row, + width): lo - width < at + i row < hi
        if (a.rows == 1) {
            if (at < hi && at + a.width > lo) return true;
        } else {
            const int64_t first = std::max<int64_t>(0, floor_div(lo - a.width - at, a.row) + 1), last = std::min(a.rows - 1, -floor_div(-(hi - at), a.row) - 1);
            if (first <= last) return true;
        }
    }
    return false;
}

// True where a and b share a byte.  Exact for arrays of equal strides (slices of one buffer) and where one of
// the two is a block; other pairs whose ranges cross are taken to be apart.  A step per group at most.
inline bool overlap(const Rows &a, const Rows &b) {
    if (a.end() <= b.base || b.end() <= a.base) return false;
    if (a.block()) return meets(b, a.base, a.end());
    if (b.block()) return meets(a, b.base, b.end());
    if (a.row != b.row || a.group != b.group) return false;
    // a's interval lies i rows and j groups from b's: -a.width < apart + i row + j group < b.width
    const int64_t apart = a.base - b.base, rows = std::max(a.rows, b.rows) - 1;
    if (a.groups == 1 && b.groups == 1) return multiple_between(-a.width - apart, b.width - apart, a.row, rows);
    const int64_t reach = rows * a.row + std::max(a.width, b.width), groups = std::max(a.groups, b.groups) - 1;
    const int64_t first = std::max(-groups, floor_div(-apart - reach, a.group)), last = std::min(groups, floor_div(reach - apart, a.group) + 1);
    for (int64_t j = first; j <= last; ++j)
        if (multiple_between(-a.width - apart - j * a.group, b.width - apart - j * a.group, a.row, rows)) return true;
    return false;
}

}  // namespace liec
