// Attention over a paged cache on the matrix cores: 16-bit values, dims that
// are multiples of 8 up to 256, 16-byte aligned rows.
//
// New token i (of c) of a sequence of n entries sees entries j <= n - c + i:
//   o = sum_j p_j v_j,   p_j = exp(x_j - max) / sum,   x_j = scale q . k_j.
//
// Rows and tiles.  The heads of a group read the same keys, so a row is a
// (token, head of the group) pair, r = i * group + g, and a tile is kRows
// consecutive rows of one (sequence, kv head): a single token of a grouped
// model and a chunk of an ungrouped one fill the same matrix operand.  A wave
// holds 32 rows.
//
// Per step a wave forms S^T = K Q^T (32x32x16 products, keys down, rows
// across), so a lane owns one row: its maximum, sum and rescaling are the
// lane's own numbers (two lanes share a row, one exchange a step).  P^T then is
// already in the layout of the second operand of O^T = V^T P^T, up to an order
// of the 16 keys of a product, which V^T's reads follow; V is stored by rows
// and transposed by the LDS read.  The running maximum and sum are 32-bit; P is
// rounded to the cache's type (relative 2^-9 each, independent, below the
// output's own rounding on average).
//
// Two forms:
//   chunks  (kSplit false): 128 rows, the 4 waves share each tile of keys;
//   tokens  (kSplit true): 32 rows at most, each wave has keys of its own and
//           the waves' results are joined in LDS.  Bound by the cache's read.
//
// Work split.  A unit is one step over kUnit keys of one tile; all units of the
// call, in the order (sequence, kv head, tile, keys), are cut into equal
// contiguous ranges, one per workgroup, whatever the sequences' lengths are
// (they are read on the device).  A tile that a cut divides leaves parts
// (unnormalised sums with their maxima) that attend_join adds in order, so the
// result does not depend on timing.
#include "kv.h"
#include "mvk_internal.h"

namespace mvk {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Mma;
template <>
struct Mma<__bf16> {
    typedef __bf16 V8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x16 mul(V8 a, V8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    static constexpr uint32_t kExp = 0x7f80u;  // exponent bits: all set in infinities and not-a-numbers
};
template <>
struct Mma<_Float16> {
    typedef _Float16 V8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x16 mul(V8 a, V8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
    static constexpr uint32_t kExp = 0x7c00u;
};

// sum_{i < n} floor((a i + b) / m), by the Euclidean descent.
__device__ uint64_t floor_sum(uint64_t n, uint64_t m, uint64_t a, uint64_t b) {
    uint64_t sum = 0;
    for (;;) {
        if (a >= m) {
            sum += n * (n - 1) / 2 * (a / m);
            a %= m;
        }
        if (b >= m) {
            sum += n * (b / m);
            b %= m;
        }
        const uint64_t y = a * n + b;
        if (y < m) return sum;
        n = y / m;
        b = y % m;
        const uint64_t t = m;
        m = a;
        a = t;
    }
}

// The tiles of one sequence (the same for each of its kv heads).
template <uint32_t kRows, uint32_t kUnit>
struct Tiles {
    uint32_t c, n, base, count, last;  // base: entries before the new tokens; last: units of the last tile
    uint32_t grp;
    __device__ Tiles(const SeqSpan& sp, uint32_t grp) : c(sp.c), n(sp.n), grp(grp) {
        base = n > c ? n - c : 0;
        count = (uint32_t)(((uint64_t)c * grp + kRows - 1) / kRows);
        last = (base + c + kUnit - 1) / kUnit;
    }
    // units of tile t: its last row is a row of token ((t + 1) kRows - 1) / grp
    __device__ uint32_t units(uint32_t t) const {
        if (t + 1 >= count) return last;
        return (base + (uint32_t)(((uint64_t)(t + 1) * kRows - 1) / grp) + kUnit) / kUnit;
    }
    // units of the tiles before t (t < count)
    __device__ uint32_t before(uint32_t t) const {
        if (t == 0) return 0;
        return (uint32_t)floor_sum(t, (uint64_t)grp * kUnit, kRows, (uint64_t)grp * (base + kUnit) + kRows - 1);
    }
    __device__ uint32_t all() const { return count == 0 ? 0 : before(count - 1) + last; }
};

struct TileArgs {
    Rows q, out;
    KvView kv;
    SeqView sq;
    uint32_t tokens, heads, grp;
    float sl2;      // scale log2(e), positive
    uint32_t flip;  // sign bits of a negative scale
    float inv_scale;
    float* lse;
    float* part;    // 2 parts a workgroup: kRows x kDim sums, then kRows (maximum, sum)
    uint4* split;   // per workgroup: the tile whose first part is its last (sequence, kv head, tile, parts)
    bool wide_out;  // out takes 8-byte stores of 4 16-bit values
};

__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
    const uint32_t lane = threadIdx.x & 63;
#pragma unroll
    for (uint32_t s = 1; s < 64; s <<= 1) {
        const uint32_t y = (uint32_t)__shfl_up((int)x, s);
        if (lane >= s) x += y;
    }
    return x;
}

// What a workgroup begins with.
struct Start {
    uint32_t s, kh, tile, unit, left;  // left: units of its range
    uint32_t total;
};

// First unit of workgroup w's range of `total` units in `groups` ranges.
__device__ __forceinline__ uint32_t range_at(uint32_t w, uint32_t total, uint32_t groups) {
    const uint32_t q = total / groups, r = total % groups;
    return w * q + min(w, r);
}
// The workgroup whose range holds unit x.
__device__ __forceinline__ uint32_t range_of(uint32_t x, uint32_t total, uint32_t groups) {
    const uint32_t q = total / groups, r = total % groups;
    if (x < r * (q + 1)) return x / (q + 1);
    return r + (x - r * (q + 1)) / q;
}

// Every wave by itself: the units of all sequences, and where range w begins.
template <uint32_t kRows, uint32_t kUnit>
__device__ __forceinline__ Start find_start(const TileArgs& a, uint32_t w, uint32_t groups) {
    const uint32_t lane = threadIdx.x & 63, hk = a.kv.heads;
    Start st = {};
    uint32_t first = 0;  // units of sequence `lane`: kept, as most calls have at most 64 sequences
    for (uint32_t s0 = 0; s0 < a.sq.count; s0 += 64) {
        const uint32_t s = s0 + lane;
        uint32_t u = 0;
        if (s < a.sq.count) u = Tiles<kRows, kUnit>(seq_span(a.sq, a.kv.shift, s, a.tokens), a.grp).all() * hk;
        if (s0 == 0) first = u;
        st.total += (uint32_t)__shfl((int)wave_scan(u), 63);
    }
    const uint32_t x = range_at(w, st.total, groups);
    st.left = range_at(w + 1, st.total, groups) - x;
    if (st.left == 0) return st;
    uint32_t seen = 0;
    for (uint32_t s0 = 0; s0 < a.sq.count; s0 += 64) {
        const uint32_t s = s0 + lane;
        uint32_t u = first;
        if (s0) {
            u = 0;
            if (s < a.sq.count) u = Tiles<kRows, kUnit>(seq_span(a.sq, a.kv.shift, s, a.tokens), a.grp).all() * hk;
        }
        const uint32_t incl = wave_scan(u);
        const uint64_t past = __ballot(seen + incl > x);
        if (past) {
            const int at = __ffsll((unsigned long long)past) - 1;
            st.s = s0 + (uint32_t)at;
            const uint32_t us = (uint32_t)__shfl((int)u, at), before = seen + (uint32_t)__shfl((int)incl, at) - us;
            const uint32_t per = us / hk, in = x - before;
            st.kh = in / per;
            const uint32_t rem = in % per;
            const Tiles<kRows, kUnit> t(seq_span(a.sq, a.kv.shift, st.s, a.tokens), a.grp);
            // the last tile whose units begin at or before rem: 64 candidates at a time
            uint32_t lo = 0, hi = t.count;
            while (hi - lo > 1) {
                const uint32_t step = (hi - lo + 63) / 64, cand = lo + lane * step;
                const uint64_t ok = __ballot(cand < hi && t.before(cand) <= rem);
                const uint32_t k = (uint32_t)__popcll(ok) - 1;  // (lane 0 always: before(lo) <= rem)
                lo += k * step;
                hi = min(hi, lo + step);
            }
            st.tile = lo;
            st.unit = rem - t.before(lo);
            return st;
        }
        seen += (uint32_t)__shfl((int)incl, 63);
    }
    st.left = 0;  // (not reached: the range begins below the total)
    return st;
}

// Granules (8 values) of a row in LDS, permuted so that the reads below meet
// every bank once: K is read granule by granule down the rows, V in blocks of 4
// rows by 2 granules.
template <uint32_t kDim>
__device__ __forceinline__ uint32_t k_at(uint32_t row, uint32_t g) {
    constexpr uint32_t G = kDim / 8;
    return row * G + (g ^ (row & (G < 16 ? G - 1 : 15)));
}
template <uint32_t kDim>
__device__ __forceinline__ uint32_t v_at(uint32_t row, uint32_t g) {
    constexpr uint32_t G = kDim / 8;
    return row * G + (g ^ (G < 16 ? ((row >> 1) & 3) * 2 : (row & 7) * 2));
}

__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The state of a wave's 32 rows: lane l has row l % 32 (l / 32: which half of
// the keys of a block, and of the dims of a product, it holds).
template <typename T, uint32_t kDim>
struct WaveRows {
    typedef typename Mma<T>::V8 V8;
    V8 q[kDim / 16];
    f32x16 o[kDim / 32];  // O^T: register i of tile d: dim 32 d + 8 (i / 4) + 4 (l / 32) + i % 4
    float m, l;           // maximum of q . k so far; this lane's part of the sum
    uint32_t lim;         // entries that the row sees

    // One step over 32 kBlocks keys, the first of them entry j0, in LDS.
    template <uint32_t kBlocks>
    __device__ __forceinline__ void step(const u32x4* lk, const u32x4* lv, uint32_t j0, bool masked, float sl2) {
        const uint32_t lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
        f32x16 s[kBlocks];
#pragma unroll
        for (uint32_t b = 0; b < kBlocks; ++b) {
            s[b] = f32x16{};
#pragma unroll
            for (uint32_t t = 0; t < kDim / 16; ++t) {
                const V8 k = __builtin_bit_cast(V8, lk[k_at<kDim>(32 * b + col, 2 * t + half)]);
                s[b] = Mma<T>::mul(k, q[t], s[b]);
            }
        }
        if (masked) {
#pragma unroll
            for (uint32_t b = 0; b < kBlocks; ++b)
#pragma unroll
                for (uint32_t i = 0; i < 16; ++i)
                    if (j0 + 32 * b + 8 * (i / 4) + 4 * half + i % 4 >= lim) s[b][i] = -INFINITY;
        }
        float top = m;
#pragma unroll
        for (uint32_t b = 0; b < kBlocks; ++b)
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
        top = max_halves(top);
        // nothing but -inf so far: sums stay zero instead of inf - inf
        const float base = top == -INFINITY ? 0.f : top * sl2;
        if (__any(top != m)) {
            const float a = __builtin_amdgcn_exp2f(m * sl2 - base);
            l *= a;
#pragma unroll
            for (uint32_t d = 0; d < kDim / 32; ++d)
#pragma unroll
                for (uint32_t i = 0; i < 16; ++i) o[d][i] *= a;
        }
        m = top;
#pragma unroll
        for (uint32_t b = 0; b < kBlocks; ++b)
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) {
                s[b][i] = __builtin_amdgcn_exp2f(s[b][i] * sl2 - base);
                l += s[b][i];
            }
        uint32_t bad = 0;
#pragma unroll
        for (uint32_t t = 0; t < 2 * kBlocks; ++t) {
            V8 p;
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) p[i] = (T)s[t / 2][8 * (t % 2) + i];
            // keys 16 t + 4 half + 0..3 and 16 t + 8 + 4 half + 0..3, as p has them
            const uint32_t r = 16 * t + 4 * half + (lane & 15) / 4;
#pragma unroll
            for (uint32_t d = 0; d < kDim / 32; ++d) {
                const uint32_t g = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
                s16x4 v[2];
#pragma unroll
                for (uint32_t w = 0; w < 2; ++w) {
                    const u32x4* at = lv + v_at<kDim>(r + 8 * w, g);
                    v[w] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) s16x4*)((const s16x4*)at + (lane & 1)));
                }
                if (masked) {
                    // 0 * inf is not 0: infinities and not-a-numbers are taken out here, see below
#pragma unroll
                    for (uint32_t w = 0; w < 2; ++w)
#pragma unroll
                        for (uint32_t e = 0; e < 4; ++e)
                            if (((uint32_t)v[w][e] & Mma<T>::kExp) == Mma<T>::kExp) {
                                v[w][e] = 0;
                                bad = 1;
                            }
                }
                const V8 vv = __builtin_bit_cast(V8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
                o[d] = Mma<T>::mul(vv, p, o[d]);
            }
        }
        if (masked && __any(bad)) {
            // the rows that see such a value get p v, the others nothing
            for (uint32_t k = 0; k < 32 * kBlocks; ++k) {
                const uint32_t b = k / 32, i = 4 * ((k % 32) / 8) + k % 4, owner = (k % 8) / 4;
                float p = 0.f;
#pragma unroll
                for (uint32_t u = 0; u < 16 * kBlocks; ++u)
                    if (u == 16 * b + i) p = s[u / 16][u % 16];
                p = __shfl(p, (int)(col + 32 * owner));
                if (j0 + k >= lim) continue;
                const T* row = (const T*)lv;
#pragma unroll
                for (uint32_t d = 0; d < kDim / 32; ++d)
#pragma unroll
                    for (uint32_t u = 0; u < 16; ++u) {
                        const uint32_t e = 32 * d + 8 * (u / 4) + 4 * half + u % 4;
                        const T x = row[8 * v_at<kDim>(k, e / 8) + e % 8];
                        if ((__builtin_bit_cast(uint16_t, x) & Mma<T>::kExp) == Mma<T>::kExp) o[d][u] += p * (float)x;
                    }
            }
        }
    }
};

// kBlocks: 32-key blocks of one tile of keys in LDS (shared, or one wave's).
template <typename T, uint32_t kDim, bool kSplit>
struct Shape {
    static constexpr uint32_t kThreads = 256;
    static constexpr uint32_t kRows = kSplit ? 32 : 128;
    static constexpr uint32_t kBlocks = kSplit ? 1 : 2;
    static constexpr uint32_t kKeys = 32 * kBlocks;                       // keys of one LDS tile
    static constexpr uint32_t kUnit = kSplit ? 4 * kKeys : kKeys;         // keys of one unit
    static constexpr uint32_t kLoaders = kSplit ? 64 : kThreads;          // threads that fill a tile
    static constexpr uint32_t kGranules = kKeys * (kDim / 8);             // of K, and of V
    static constexpr uint32_t kPer = kGranules / kLoaders;                // granules a thread
    static constexpr uint32_t kLds = (kSplit ? 4 : 2) * 2 * kGranules;    // granules: a wave's, or two stages
    static constexpr uint32_t kPart = kRows * kDim + 2 * kRows;           // floats of a part
};

// Four consecutive values of a row of the output.
__device__ __forceinline__ void put4(const TileArgs& a, size_t at, f32x4 x) {
    if (a.wide_out) {
        typedef __bf16 B4 __attribute__((ext_vector_type(4)));
        typedef _Float16 H4 __attribute__((ext_vector_type(4)));
        u32x2 v;
        if (a.out.type == MVK_TYPE_BF16) v = __builtin_bit_cast(u32x2, __builtin_convertvector(x, B4));
        else v = __builtin_bit_cast(u32x2, __builtin_convertvector(x, H4));
        *(u32x2*)((uint16_t*)a.out.p + at) = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) store_as(a.out.p, a.out.type, at + i, x[i], a.inv_scale);
}

template <typename T, uint32_t kDim, bool kSplit>
__global__ __launch_bounds__(256, kDim > 128 ? 1 : 2) void attend_tile(TileArgs a) {
    typedef Shape<T, kDim, kSplit> Sh;
    typedef typename Mma<T>::V8 V8;
    __shared__ u32x4 lds[Sh::kLds];
    __shared__ float red[4][32][2];
    const uint32_t tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 31, half = lane >> 5;
    const uint32_t dim = a.kv.dim, live = dim / 8;  // granules of a row that hold data
    // consecutive ranges on one XCD, whose L2 then holds the keys they share
    const uint32_t groups = gridDim.x, xcds = groups % 8 == 0 ? 8 : 1;
    const uint32_t w = (blockIdx.x % xcds) * (groups / xcds) + blockIdx.x / xcds;
    Start st = find_start<Sh::kRows, Sh::kUnit>(a, w, groups);
    if (tid == 0) a.split[w] = uint4{0, 0, 0, 0};
    const uint32_t loader = kSplit ? lane : tid;
    const uint32_t lg = loader % (kDim / 8), lr = loader / (kDim / 8);        // first granule of this thread
    constexpr uint32_t kRowStep = Sh::kLoaders / (kDim / 8);                  // rows between its granules
    u32x4* const mine = kSplit ? lds + wave * 2 * Sh::kGranules : lds;

    uint32_t done = 0;
    while (done < st.left) {
        const SeqSpan sp = seq_span(a.sq, a.kv.shift, st.s, a.tokens);
        const Tiles<Sh::kRows, Sh::kUnit> tiles(sp, a.grp);
        const uint32_t units = tiles.units(st.tile);
        const uint32_t u0 = st.unit, u1 = min(units, u0 + (st.left - done));

        // rows
        const uint32_t rows = sp.c * a.grp, row0 = st.tile * Sh::kRows + (kSplit ? 0 : 32 * wave);
        const uint32_t row = row0 + col, known = min(row, rows - 1);
        const bool valid = row < rows;
        const uint32_t tok = sp.q0 + known / a.grp, head = st.kh * a.grp + known % a.grp;
        WaveRows<T, kDim> x;
        {
            const int64_t see = (int64_t)sp.n - sp.c + known / a.grp + 1;
            x.lim = see > 0 ? (uint32_t)see : 0u;
            const T* qr = (const T*)a.q.p + (size_t)tok * a.q.token + (size_t)head * a.q.head;
#pragma unroll
            for (uint32_t t = 0; t < kDim / 16; ++t) {
                u32x4 v = {0, 0, 0, 0};
                const uint32_t g = 2 * t + half;
                if (valid && g < live) v = *(const u32x4*)(qr + 8 * g) ^ a.flip;
                x.q[t] = __builtin_bit_cast(V8, v);
            }
#pragma unroll
            for (uint32_t d = 0; d < kDim / 32; ++d) x.o[d] = f32x16{};
            x.m = -INFINITY;
            x.l = 0.f;
        }
        // limits of the wave's rows: rows are in order, so lane 0 sees least
        const uint32_t lim_lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)x.lim);
        const uint32_t lim_hi = (uint32_t)__builtin_amdgcn_readlane((int)x.lim, 31);
        const bool idle = !kSplit && row0 >= rows;  // a wave without rows

        const T* const kb = (const T*)a.kv.K + (size_t)st.kh * a.kv.kh;
        const T* const vb = (const T*)a.kv.V + (size_t)st.kh * a.kv.vh;
        u32x4 rk[Sh::kPer], rv[Sh::kPer];
        uint32_t pg[Sh::kPer];
        const uint32_t mask = (1u << a.kv.shift) - 1;
        const uint32_t first = u0 * Sh::kUnit + (kSplit ? wave * Sh::kKeys : 0);
        const uint32_t stop = min(u1 * Sh::kUnit, sp.n);  // entries at and beyond it are not needed
        // entries beyond the last are loaded as the last (and masked): no address leaves the sequence
        auto pages = [&](uint32_t j0) {
            if (j0 < stop) {
#pragma unroll
                for (uint32_t i = 0; i < Sh::kPer; ++i) pg[i] = seq_page(a.sq, a.kv, st.s, min(j0 + lr + i * kRowStep, sp.n - 1));
            }
        };
        auto load = [&](uint32_t j0) {
            if (j0 < stop) {
#pragma unroll
                for (uint32_t i = 0; i < Sh::kPer; ++i) {
                    const uint32_t e = min(j0 + lr + i * kRowStep, sp.n - 1) & mask;
                    rk[i] = rv[i] = u32x4{0, 0, 0, 0};
                    if (lg < live) {
                        rk[i] = *(const u32x4*)(kb + pg[i] * a.kv.kp + e * a.kv.ke + 8 * lg);
                        rv[i] = *(const u32x4*)(vb + pg[i] * a.kv.vp + e * a.kv.ve + 8 * lg);
                    }
                }
            }
        };
        auto store = [&](u32x4* to) {
#pragma unroll
            for (uint32_t i = 0; i < Sh::kPer; ++i) {
                to[k_at<kDim>(lr + i * kRowStep, lg)] = rk[i];
                to[Sh::kGranules + v_at<kDim>(lr + i * kRowStep, lg)] = rv[i];
            }
        };
        pages(first);
        load(first);
        pages(first + Sh::kUnit);
        uint32_t stage = 0;
        for (uint32_t j0 = first; j0 < stop; j0 += Sh::kUnit) {
            u32x4* const buf = kSplit ? mine : mine + stage * 2 * Sh::kGranules;
            store(buf);
            if (kSplit) {
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            } else {
                __syncthreads();  // the other stage is free: every wave has passed its step
            }
            load(j0 + Sh::kUnit);
            pages(j0 + 2 * Sh::kUnit);
            if (!idle && j0 < lim_hi)
                x.template step<Sh::kBlocks>(buf, buf + Sh::kGranules, j0, j0 + Sh::kKeys > lim_lo, a.sl2);
            if (kSplit) {
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
            stage ^= 1;
        }

        // the rows' results
        const bool whole = u0 == 0 && u1 == units;
        float* const part = a.part + (size_t)(2 * w + (u0 == 0 ? 1 : 0)) * Sh::kPart;
        float l = sum_halves(x.l);
        if (kSplit) {
            // join the waves: the common maximum, then sums of the rescaled rows
            if (lane < 32) red[wave][lane][0] = x.m, red[wave][lane][1] = l;
            __syncthreads();
            float m = red[0][col][0];
#pragma unroll
            for (uint32_t i = 1; i < 4; ++i) m = fmaxf(m, red[i][col][0]);
            const float base = m == -INFINITY ? 0.f : m * a.sl2;
            const float f = __builtin_amdgcn_exp2f(x.m * a.sl2 - base);
            float* const all = (float*)lds;  // wave, row, dim (rows kDim + 4 apart would cost LDS that is not there)
            float* const own = all + (size_t)wave * 32 * kDim + col * kDim;
            const uint32_t n32 = min(rows - row0, 32u);
            if (col < n32) {
#pragma unroll
                for (uint32_t d = 0; d < kDim / 32; ++d)
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        const uint32_t e = 32 * d + 8 * i + 4 * half;
                        f32x4 y;
#pragma unroll
                        for (uint32_t k = 0; k < 4; ++k) y[k] = x.o[d][4 * i + k] * f;
                        *(f32x4*)(own + ((e / 4) ^ (col & 7)) * 4) = y;
                    }
            }
            __syncthreads();
            for (uint32_t i = tid; i < n32 * (kDim / 4); i += 256) {
                const uint32_t r = i / (kDim / 4), g = i % (kDim / 4);
                if (4 * g >= dim) continue;
                f32x4 y = {0.f, 0.f, 0.f, 0.f};
                float ls = 0.f, mr = red[0][r][0];
#pragma unroll
                for (uint32_t v = 1; v < 4; ++v) mr = fmaxf(mr, red[v][r][0]);
                const float b2 = mr == -INFINITY ? 0.f : mr * a.sl2;
#pragma unroll
                for (uint32_t v = 0; v < 4; ++v) {
                    y += *(const f32x4*)(all + (size_t)v * 32 * kDim + r * kDim + (g ^ (r & 7)) * 4);
                    ls += red[v][r][1] * __builtin_amdgcn_exp2f(red[v][r][0] * a.sl2 - b2);
                }
                if (whole) {
                    const uint32_t rr = row0 + r, t2 = sp.q0 + rr / a.grp, h2 = st.kh * a.grp + rr % a.grp;
                    const float inv = ls > 0.f ? 1.f / ls : ls == 0.f ? 0.f : ls;
                    put4(a, (size_t)t2 * a.out.token + (size_t)h2 * a.out.head + 4 * g, y * inv);
                    if (a.lse && g == 0)
                        a.lse[(size_t)t2 * a.heads + h2] =
                            ls > 0.f ? (mr * a.sl2 + log2f(ls)) * kLn2 : ls == 0.f ? -INFINITY : ls;
                } else {
                    *(f32x4*)(part + r * kDim + 4 * g) = y;
                    if (g == 0) part[Sh::kRows * kDim + 2 * r] = mr, part[Sh::kRows * kDim + 2 * r + 1] = ls;
                }
            }
        } else if (valid) {
            const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
            const size_t at = (size_t)tok * a.out.token + (size_t)head * a.out.head;
            const uint32_t r = 32 * wave + col;
#pragma unroll
            for (uint32_t d = 0; d < kDim / 32; ++d)
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {
                    const uint32_t e = 32 * d + 8 * i + 4 * half;
                    if (e >= dim) continue;
                    f32x4 y;
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) y[k] = x.o[d][4 * i + k];
                    if (whole) put4(a, at + e, y * inv);
                    else *(f32x4*)(part + (size_t)r * kDim + e) = y;
                }
            if (half == 0) {
                if (!whole) part[Sh::kRows * kDim + 2 * r] = x.m, part[Sh::kRows * kDim + 2 * r + 1] = l;
                else if (a.lse)
                    a.lse[(size_t)tok * a.heads + head] =
                        l > 0.f ? (x.m * a.sl2 + log2f(l)) * kLn2 : l == 0.f ? -INFINITY : l;
            }
        }
        if (tid == 0 && u0 == 0 && !whole) {
            // the tile goes on in the next ranges
            const uint32_t at = range_at(w, st.total, groups) + done;
            a.split[w] = uint4{st.s, st.kh, st.tile, range_of(at + units - 1, st.total, groups) - w};
        }
        __syncthreads();  // LDS is free again

        done += u1 - u0;
        st.unit = 0;
        if (++st.tile == tiles.count) {
            st.tile = 0;
            if (++st.kh == a.kv.heads) {
                st.kh = 0;
                if (done < st.left)
                    do ++st.s;
                    while (st.s + 1 < a.sq.count && seq_span(a.sq, a.kv.shift, st.s, a.tokens).c == 0);
            }
        }
    }
}

// Adds the parts of the tiles that a cut divides, in order: workgroup (w, y)
// has rows y kJoinRows .. of the tile whose first part is the last of range w.
constexpr uint32_t kJoinRows = 8;
template <typename T, uint32_t kDim, bool kSplit>
__global__ __launch_bounds__(256) void attend_join(TileArgs a) {
    typedef Shape<T, kDim, kSplit> Sh;
    const uint32_t w = blockIdx.x;
    const uint4 d = a.split[w];
    if (d.w == 0) return;
    const SeqSpan sp = seq_span(a.sq, a.kv.shift, d.x, a.tokens);
    const uint32_t rows = sp.c * a.grp, row0 = d.z * Sh::kRows;
    for (uint32_t i = threadIdx.x; i < kJoinRows * (kDim / 4); i += 256) {
        const uint32_t r = blockIdx.y * kJoinRows + i / (kDim / 4), g = i % (kDim / 4), row = row0 + r;
        if (row >= rows || 4 * g >= a.kv.dim) continue;
        float m = -INFINITY, l = 0.f;
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
        for (uint32_t k = 0; k <= d.w; ++k) {
            const float* p = a.part + (size_t)(2 * (w + k) + (k == 0 ? 1 : 0)) * Sh::kPart;
            const float mk = p[Sh::kRows * kDim + 2 * r], lk = p[Sh::kRows * kDim + 2 * r + 1];
            const f32x4 yk = *(const f32x4*)(p + (size_t)r * kDim + 4 * g);
            const float top = fmaxf(m, mk), base = top == -INFINITY ? 0.f : top * a.sl2;
            const float fa = __builtin_amdgcn_exp2f(m * a.sl2 - base), fb = __builtin_amdgcn_exp2f(mk * a.sl2 - base);
            m = top;
            l = l * fa + lk * fb;
            y = y * fa + yk * fb;
        }
        const uint32_t t = sp.q0 + row / a.grp, h = d.y * a.grp + row % a.grp;
        const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
        put4(a, (size_t)t * a.out.token + (size_t)h * a.out.head + 4 * g, y * inv);
        if (a.lse && g == 0)
            a.lse[(size_t)t * a.heads + h] = l > 0.f ? (m * a.sl2 + log2f(l)) * kLn2 : l == 0.f ? -INFINITY : l;
    }
}

// Collected weights: a workgroup owns kWeightKeys entries of one (sequence, kv
// head), 32 a wave, and adds the probabilities of all rows that see them, in
// order: S = Q K^T (rows down, keys across, so that a lane sums its own key),
// p = exp(scale S - lse).  K is read once; each wave reads the rows for itself.
constexpr uint32_t kWeightKeys = 128;
template <typename T, uint32_t kDim>
__global__ __launch_bounds__(256) void weights_tile(TileArgs a, const float* __restrict__ lse, const float* w_in,
                                                    float* w_out, size_t w_seq, size_t w_head) {
    typedef typename Mma<T>::V8 V8;
    __shared__ float row_lse[4][32];
    __shared__ uint32_t row_lim[4][32];
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const uint32_t kh = blockIdx.y, s = blockIdx.z, live = a.kv.dim / 8;
    const SeqSpan sp = seq_span(a.sq, a.kv.shift, s, a.tokens);
    const uint32_t j0 = blockIdx.x * kWeightKeys + 32 * wave;
    if (j0 >= sp.n) return;  // no barrier below spans waves
    const int64_t base = (int64_t)sp.n - sp.c;
    const uint32_t j = j0 + col, jc = min(j, sp.n - 1);
    V8 k[kDim / 16];
    {
        const size_t page = seq_page(a.sq, a.kv, s, jc), at = jc & ((1u << a.kv.shift) - 1);
        const T* kr = (const T*)a.kv.K + page * a.kv.kp + kh * a.kv.kh + at * a.kv.ke;
#pragma unroll
        for (uint32_t t = 0; t < kDim / 16; ++t) {
            u32x4 v = {0, 0, 0, 0};
            const uint32_t g = 2 * t + half;
            if (g < live) v = *(const u32x4*)(kr + 8 * g);
            k[t] = __builtin_bit_cast(V8, v);
        }
    }
    const uint32_t rows = sp.c * a.grp;
    // rows of the first token that sees entry j0, from a whole 32 on
    uint32_t r0 = j0 > base ? (uint32_t)((int64_t)j0 - base) * a.grp / 32 * 32 : 0u;
    float sum = 0.f;
    u32x4 q[kDim / 16];
    float z = 0.f;
    uint32_t lim = 0;
    auto load = [&](uint32_t r) {
        const uint32_t row = r + col;
        const uint32_t tok = row / a.grp, head = kh * a.grp + row % a.grp;
        z = INFINITY;
        lim = 0;
#pragma unroll
        for (uint32_t t = 0; t < kDim / 16; ++t) q[t] = u32x4{0, 0, 0, 0};
        if (row < rows) {
            const int64_t see = base + tok + 1;
            lim = see > 0 ? (uint32_t)see : 0u;
            z = lse[(size_t)(sp.q0 + tok) * a.heads + head] * kLog2e;
            if (z == -INFINITY) z = INFINITY;  // a row without a sum gives nothing
            const T* qr = (const T*)a.q.p + (size_t)(sp.q0 + tok) * a.q.token + (size_t)head * a.q.head;
#pragma unroll
            for (uint32_t t = 0; t < kDim / 16; ++t) {
                const uint32_t g = 2 * t + half;
                if (g < live) q[t] = *(const u32x4*)(qr + 8 * g) ^ a.flip;
            }
        }
    };
    if (r0 < rows) load(r0);
    for (; r0 < rows; r0 += 32) {
        if (half == 0) row_lse[wave][col] = z, row_lim[wave][col] = lim;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        f32x16 x = {};
#pragma unroll
        for (uint32_t t = 0; t < kDim / 16; ++t) x = Mma<T>::mul(__builtin_bit_cast(V8, q[t]), k[t], x);
        const bool masked = j0 + 32 > (uint32_t)__builtin_amdgcn_readfirstlane((int)lim) || r0 + 32 > rows;
        if (r0 + 32 < rows) load(r0 + 32);
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i) {
            const uint32_t r = 8 * (i / 4) + 4 * half + i % 4;
            float p = __builtin_amdgcn_exp2f(x[i] * a.sl2 - row_lse[wave][r]);
            if (masked && j >= row_lim[wave][r]) p = 0.f;
            sum += p;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    sum = sum_halves(sum);
    if (half == 0 && j < sp.n) {
        const size_t o = (size_t)s * w_seq + (size_t)kh * w_head + j;
        w_out[o] = ((int64_t)j < base && w_in ? w_in[o] : 0.f) + sum;
    }
}

constexpr uint32_t kGroups = 512;  // two workgroups a compute unit

template <typename T, uint32_t kDim, bool kSplit>
size_t part_floats() {
    return (size_t)2 * kGroups * Shape<T, kDim, kSplit>::kPart;
}

template <typename T, uint32_t kDim, bool kSplit>
hipError_t launch_shape(TileArgs a, void* ws, hipStream_t s) {
    a.split = (uint4*)ws;
    a.part = (float*)((char*)ws + kGroups * sizeof(uint4));
    hipLaunchKernelGGL((attend_tile<T, kDim, kSplit>), dim3(kGroups), dim3(256), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((attend_join<T, kDim, kSplit>), dim3(kGroups, Shape<T, kDim, kSplit>::kRows / kJoinRows),
                       dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const TileArgs& a, bool split, void* ws, hipStream_t s) {
    const uint32_t d = a.kv.dim;
    if (split) {
        if (d <= 64) return launch_shape<T, 64, true>(a, ws, s);
        if (d <= 128) return launch_shape<T, 128, true>(a, ws, s);
        return launch_shape<T, 256, true>(a, ws, s);
    }
    if (d <= 64) return launch_shape<T, 64, false>(a, ws, s);
    if (d <= 128) return launch_shape<T, 128, false>(a, ws, s);
    return launch_shape<T, 256, false>(a, ws, s);
}

inline bool in16(const void* p, size_t a, size_t b, size_t c) { return (uintptr_t)p % 16 == 0 && (a | b | c) % 8 == 0; }

}  // namespace

bool attend_tile_fits(const Rows& q, uint32_t tokens, uint32_t heads, const KvView& kv, const SeqView& sq) {
    if ((q.type != MVK_TYPE_BF16 && q.type != MVK_TYPE_F16) || kv.dim % 8 || kv.dim > 256 || tokens == 0) return false;
    if (!in16(q.p, q.token, q.head, 0) || !in16(kv.K, kv.kp, kv.kh, kv.ke) || !in16(kv.V, kv.vp, kv.vh, kv.ve))
        return false;
    // units are counted in 32 bits (64 keys a unit at least, 32 rows a tile)
    const uint64_t grp = heads / kv.heads, tiles = (tokens * grp) / 32 + sq.count;
    const uint64_t units = (((uint64_t)sq.width << kv.shift) + tokens) / 64 + 1;
    return tiles < (1ull << 31) / units / kv.heads;
}

size_t attend_tile_bytes(const KvView& kv, bool split) {
    const uint32_t dim = kv.dim <= 64 ? 64 : kv.dim <= 128 ? 128 : 256, rows = split ? 32 : 128;
    return kGroups * sizeof(uint4) + (size_t)2 * kGroups * (rows * dim + 2 * rows) * sizeof(float);
}

bool attend_tile_split(uint32_t max_new, uint32_t heads, const KvView& kv) {
    return (uint64_t)max_new * (heads / kv.heads) <= 32;
}

namespace {

TileArgs tile_args(const Rows& q, uint32_t tokens, uint32_t heads, const KvView& kv, const SeqView& sq, float scale) {
    TileArgs a = {};
    a.q = q, a.kv = kv, a.sq = sq, a.tokens = tokens, a.heads = heads, a.grp = heads / kv.heads;
    // the sign goes to q; a scale of zero as one that no score survives, so that masked places stay at -inf
    const float mag = scale < 0 ? -scale : scale;
    a.sl2 = mag < 1e-30f ? 1e-30f : mag * kLog2e;
    a.flip = scale < 0 ? 0x80008000u : 0u;
    return a;
}

}  // namespace

hipError_t launch_weights_tile(const Rows& q, uint32_t tokens, uint32_t heads, const KvView& kv, const SeqView& sq,
                               float scale, const float* lse, const float* w_in, float* w_out, size_t w_seq,
                               size_t w_head, hipStream_t s) {
    const TileArgs a = tile_args(q, tokens, heads, kv, sq, scale);
    const uint64_t cap = (uint64_t)sq.width << kv.shift;
    const dim3 grid((uint32_t)((cap + kWeightKeys - 1) / kWeightKeys), kv.heads, sq.count);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, lse, w_in, w_out, w_seq, w_head);
        return hipGetLastError();
    };
    const uint32_t d = kv.dim <= 64 ? 0 : kv.dim <= 128 ? 1 : 2;
    if (q.type == MVK_TYPE_BF16)
        return d == 0 ? go(weights_tile<__bf16, 64>) : d == 1 ? go(weights_tile<__bf16, 128>) : go(weights_tile<__bf16, 256>);
    return d == 0 ? go(weights_tile<_Float16, 64>) : d == 1 ? go(weights_tile<_Float16, 128>) : go(weights_tile<_Float16, 256>);
}

hipError_t launch_attend_tile(const Rows& q, uint32_t tokens, uint32_t heads, const KvView& kv, const SeqView& sq,
                              float scale, const Rows& out, float inv_scale, float* lse, bool split, void* ws,
                              hipStream_t s) {
    TileArgs a = tile_args(q, tokens, heads, kv, sq, scale);
    a.out = out;
    a.inv_scale = inv_scale, a.lse = lse;
    a.wide_out = (out.type == MVK_TYPE_BF16 || out.type == MVK_TYPE_F16) && (uintptr_t)out.p % 8 == 0 &&
                 (out.token | out.head) % 4 == 0;
    return q.type == MVK_TYPE_BF16 ? launch_type<__bf16>(a, split, ws, s) : launch_type<_Float16>(a, split, ws, s);
}

}  // namespace mvk
