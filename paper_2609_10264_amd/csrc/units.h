// The work split of attention on the matrix cores: tiles of rows, their units,
// and how many units a call can have (attention_tile.hip).
#pragma once
#include <stdint.h>

#ifndef MVK_HD
#define MVK_HD __host__ __device__ __forceinline__
#endif

namespace mvk {

// sum_{i < n} floor((a i + b) / m), by the Euclidean descent; a n + b and the
// sum are below 2^32 (units_fit).
MVK_HD uint32_t floor_sum(uint32_t n, uint32_t m, uint32_t a, uint32_t b) {
    uint32_t sum = 0;
#pragma unroll 1
    for (;;) {
        const uint32_t qa = a / m, qb = b / m;
        sum += (uint32_t)((uint64_t)n * (n - 1) / 2) * qa + n * qb;
        a -= qa * m;
        b -= qb * m;
        const uint32_t y = a * n + b;
        if (y < m) return sum;
        n = y / m;
        b = y - n * m;
        const uint32_t t = m;
        m = a;
        a = t;
    }
}

// The tiles of one sequence of c new tokens and n entries (the same for each of
// its kv heads; grp rows a token).  A tile has a unit for every kUnit keys that
// its rows see (one at least) and, before them, kExtra units without keys: what
// its beginning and end cost besides.
template <uint32_t kRows, uint32_t kUnit, uint32_t kExtra>
struct Tiles {
    uint32_t c, n, base, count, last;  // base: entries before the new tokens; last: units of the last tile, the most
    uint32_t grp;
    MVK_HD Tiles(uint32_t c, uint32_t n, uint32_t grp) : c(c), n(n), grp(grp) {
        base = n > c ? n - c : 0;
        count = (c * grp + kRows - 1) / kRows;
        last = ((n > 1 ? n : 1) + kUnit - 1) / kUnit + kExtra;
    }
    // units of tile t: its last row is a row of token ((t + 1) kRows - 1) / grp (with more
    // new tokens than entries, token i is counted with min(i + 1, n), of which it sees fewer)
    MVK_HD uint32_t units(uint32_t t) const {
        if (t + 1 >= count) return last;
        const uint32_t u = (base + ((t + 1) * kRows - 1) / grp + kUnit) / kUnit + kExtra;
        return u < last ? u : last;
    }
    // units of the tiles before t (t < count)
    MVK_HD uint32_t before(uint32_t t) const {
        if (t == 0) return 0;
        uint32_t rising = t;  // (the tiles beyond them have `last`: only with more new tokens than entries)
        if (c > n) {
            const uint32_t r = (last - kExtra) * kUnit * grp / kRows;
            rising = r < t ? r : t;
        }
        return floor_sum(rising, grp * kUnit, kRows, grp * (base + kUnit) + kRows - 1) + rising * kExtra +
               (t - rising) * last;
    }
    MVK_HD uint32_t all() const { return count == 0 ? 0 : before(count - 1) + last; }
};

// May the units of a call be counted in 32 bits, whatever its lengths and starts are (as
// long as the starts ascend)?  tokens rows of new tokens, cap: entries a sequence can have.
// A sequence has at most grp c / kRows + 1 tiles, and a tile cap / kUnit + 1 units with keys.
template <uint32_t kRows, uint32_t kUnit, uint32_t kExtra>
inline bool units_fit(uint64_t tokens, uint64_t grp, uint64_t kv_heads, uint64_t count, uint64_t cap) {
    if (grp * (cap + 2 * kUnit) + 2 * kRows >= (1ull << 32)) return false;  // (below 2^62: both factors are below 2^31)
    const uint64_t tiles = tokens * grp / kRows + count, units = cap / kUnit + 1 + kExtra;
    return tiles <= 0xfffffffeull / units / kv_heads;
}

}  // namespace mvk
