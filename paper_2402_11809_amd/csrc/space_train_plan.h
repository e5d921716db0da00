// Host arithmetic of the losses and of the gradient lists: which buffers may lie where, and how a list of gradients is cut.
// Plain C++, so that it can be checked without a GPU.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace space {

// Whether rows of `cols` elements of `bytes` at x (stride xs elements) and at d (stride ds) have no byte in common.
inline bool rows_apart(uintptr_t x, int64_t xs, uintptr_t d, int64_t ds, int64_t rows, int64_t cols, size_t bytes) {
    const uintptr_t x_end = x + ((uintptr_t)(rows - 1) * xs + cols) * bytes, d_end = d + ((uintptr_t)(rows - 1) * ds + cols) * bytes;
    if (x >= d_end || d >= x_end) return true;
    // rows side by side in one buffer (the same stride, columns that do not meet) are apart all the same
    const uintptr_t off = (x < d ? d - x : x - d) / bytes % (uintptr_t)xs;
    return xs == ds && off >= (uintptr_t)cols && (uintptr_t)xs - off >= (uintptr_t)cols;
}

// Whether rows of `cols` elements of `bytes` at x (stride xs elements) have a byte of lo .. hi - 1.
inline bool rows_meet(uintptr_t x, int64_t xs, int64_t rows, int64_t cols, size_t bytes, uintptr_t lo, uintptr_t hi) {
    const uintptr_t step = (uintptr_t)xs * bytes, len = (uintptr_t)cols * bytes;
    const uintptr_t r = lo < x + len ? 0 : (lo - x - len) / step + 1;  // the first row that ends behind lo
    return r < (uintptr_t)rows && x + r * step < hi;
}

// Whether a and b, of so many bytes, have one in common (an empty range has none).
inline bool ranges_meet(uintptr_t a, uintptr_t a_bytes, uintptr_t b, uintptr_t b_bytes) {
    return a_bytes && b_bytes && (a < b ? b - a < a_bytes : a - b < b_bytes);
}

struct ByteRange {
    uintptr_t lo, hi;
    bool written;
};
// Whether no range that is written meets another one.  Sorts the ranges.
inline bool written_apart(ByteRange* r, size_t n) {
    std::sort(r, r + n, [](const ByteRange& a, const ByteRange& b) { return a.lo < b.lo; });
    uintptr_t end = 0, end_written = 0;  // of the ranges before
    for (size_t i = 0; i < n; ++i) {
        if (r[i].lo < (r[i].written ? end : end_written)) return false;
        end = std::max(end, r[i].hi);
        if (r[i].written) end_written = std::max(end_written, r[i].hi);
    }
    return true;
}

}  // namespace space
