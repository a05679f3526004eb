// Whether two sets of strided rows share memory, for the checks of the attention
// calls' arguments (host only).
#pragma once
#include <stdint.h>

#include <algorithm>

namespace mvk {

// Rows of `len` bytes at p + i*s0 + j*s1 (bytes), i < n0, j < n1, below 2^62 bytes in all.
struct RowSet {
    const void* p;
    uint64_t n0, s0, n1, s1, len;
    uint64_t begin() const { return (uint64_t)(uintptr_t)p; }
    uint64_t end() const { return begin() + (n0 - 1) * s0 + (n1 - 1) * s1 + len; }
};

// Do rows of a and b share memory?  Exact where the outer strides are the same (or one
// side has no second row to use its own), as those of parts of one buffer are; with
// others, or very many inner rows, where their extents meet.
inline bool share_memory(const RowSet& a, const RowSet& b) {
    if (!a.n0 || !a.n1 || !b.n0 || !b.n1) return false;
    if (a.end() <= b.begin() || b.end() <= a.begin()) return false;
    if (a.n0 > 1 && b.n0 > 1 && a.s0 != b.s0) return true;
    const int64_t d = (int64_t)(b.begin() - a.begin()), s0 = (int64_t)(a.n0 > 1 ? a.s0 : b.s0);
    // a's inner rows all before or behind b's in every outer row, as parts of one row are
    const int64_t ea = (int64_t)((a.n1 - 1) * a.s1 + a.len), eb = (int64_t)((b.n1 - 1) * b.s1 + b.len);
    if (s0) {
        const int64_t at = (d % s0 + s0) % s0;
        if (at >= ea && at + eb <= s0) return false;
    }
    // inner rows `x` bytes apart (b's from a's): does x + di s0 lie in (-b.len, a.len) for some rows di apart?
    auto meet = [&](int64_t x) {
        const int64_t low = -(int64_t)b.len - x;  // di s0 has to exceed it
        int64_t di = 1 - (int64_t)a.n0;
        if (s0) di = std::max(di, low / s0 - (low % s0 < 0) + 1);  // (floor and one)
        return di < (int64_t)b.n0 && di * s0 > low && x + di * s0 < (int64_t)a.len;
    };
    if (a.n1 == 1 || b.n1 == 1 || a.s1 == b.s1) {
        const int64_t s1 = (int64_t)(a.n1 > 1 ? a.s1 : b.s1);
        if ((a.n1 | b.n1) > 65536u) return true;
        for (int64_t dj = 1 - (int64_t)a.n1; dj < (int64_t)b.n1; ++dj)
            if (meet(d + dj * s1)) return true;
        return false;
    }
    if (a.n1 > 65536u / b.n1) return true;
    for (uint64_t i = 0; i < a.n1; ++i)
        for (uint64_t j = 0; j < b.n1; ++j)
            if (meet(d + (int64_t)(j * b.s1) - (int64_t)(i * a.s1))) return true;
    return false;
}

}  // namespace mvk
