// Attention over a paged cache on the matrix cores: 16-bit values, dims that
// are multiples of 8 up to 256, 16-byte aligned rows, units counted in 32 bits
// (units_fit).
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
// rounded to the cache's type, as the second product takes it (relative 2^-8 in
// bfloat16 and 2^-11 in half at most, independent of one another).  In the result
// that is 0.0015 (bfloat16) and 0.00018 (half) of its size, a little less than one
// rounding of it to the same type (0.0016, 0.00021); where the result is FIELD or
// 32-bit floats it is nearly all of the error.
//
// Two forms:
//   chunks  (kSplit false): 128 rows, the 4 waves share each tile of keys;
//   tokens  (kSplit true): 32 rows at most, each wave has keys of its own and
//           the waves' results are joined in LDS.  Bound by the cache's read.
// K and V go from memory straight to LDS, 16 bytes a lane; the order of the
// granules that the reads want comes from which granule a lane asks for.  The
// chunks form keeps two tiles, one in flight; the tokens form one, whose K half
// is asked for again as soon as S is formed and whose V half when O is.
//
// Work split.  A unit is one step over kUnit keys of one tile; all units of the
// call, in the order (sequence, kv head, tile, keys), are cut into equal
// contiguous ranges, one per workgroup, whatever the sequences' lengths are
// (they are read on the device).  A tile that a cut divides leaves parts
// (unnormalised sums with their maxima); the workgroup that counts itself last
// on it adds them in order, so the result does not depend on timing.
//
// Measured, dim 128 in bfloat16 (a large copy: 5.19 TB/s, an 8192^3 product: 1369
// TFLOP/s): tokens, 48 sequences of 130 to 32767 entries, 64 + 8 heads: 227 us, 5.33
// TB/s of cache; one token over 2048 entries of 32 heads 15 us, of which 6.5 are its
// bytes, the rest starts, first loads and joins.  Chunks, a prompt of 8192, 32 heads:
// 673 us, 816 TFLOP/s.  There the counters have the matrix cores busy in 39 % of the
// cycles, vector instructions in 43 %, both at once in 17 %, the LDS in 20 % (no
// bank conflicts), at 1.9 GHz: a wave's products, weights and reads follow one
// another, and with two waves a SIMD a third of the cycles has neither of the first.
//
// Which form: tokens where a sequence has at most 32 rows a kv head, one tile.  Both
// at 8 kv heads, tokens / chunks form in us: 32 sequences over 8000 entries, 8 rows
// 191 / 238, 32 rows 213 / 239, 64 rows 194 / 241; 4 over 30000, 16 rows 104 / 151, 64 rows
// 151 / 154; 64 over 500, 8 rows 26.6 / 27.5, 32 rows 28.5 / 28.1, 40 rows 44.8 / 29.5, 64
// rows 46.9 / 30.9; 32 over 8000, 96 rows 566 / 244.  From 33 to 64 rows long contexts
// would gain a fifth by the tokens form and short ones lose half; their lengths are
// on the device, so the bound is where no context loses.
//
// Caches held in 8 bits (a code times a power of two of its row, exact in bfloat16)
// are widened on the way to the same products.  Tokens form: a lane has a key and half
// of its dims, 16 codes a load, and widens them in the operands' registers; V goes by
// way of registers to LDS.  Chunks form: it has no registers for that while it
// computes, so the codes go straight to LDS and each wave widens its own part of a tile
// in place at the end of a step.  Measured: the 48 sequences above 161 us in E4M3 (227
// in bfloat16; 118 are its bytes), a chunk of 512 over 16000 entries with 64 + 8 heads
// 357 us (304 in bfloat16): the widening, two conversions and an LDS pass a value, is
// paid once a workgroup and tile and adds to steps that the products already fill.  I8
// takes 10 to 18 % longer than E4M3, which one instruction converts by pairs.
#include "kv.h"
#include "mvk_internal.h"
#include "quant.h"
#include "units.h"

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
    uint32_t* counters;  // one a workgroup, kCounterStride words apart: zero before and after
    bool whole_page;     // a tile of keys lies in one page, its offsets in 32 bits, and dim is kDim
    bool wide_out;  // out takes stores of 4 values at once
    bool by_16;     // codes of a cache held in 8 bits come 16 at a time
};

// Sums that stop at kTooMany: sequences whose starts do not ascend share token rows
// and may have more units together than units_fit allows for.
constexpr uint32_t kTooMany = 0xffffffffu;
__device__ __forceinline__ uint32_t add_units(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
    const uint32_t lane = threadIdx.x & 63;
#pragma unroll
    for (uint32_t s = 1; s < 64; s <<= 1) {
        const uint32_t y = (uint32_t)__shfl_up((int)x, s);
        if (lane >= s) x = add_units(x, y);
    }
    return x;
}

__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }

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
template <uint32_t kRows, uint32_t kUnit, uint32_t kExtra>
__device__ __forceinline__ Start find_start(const TileArgs& a, uint32_t w, uint32_t groups) {
    const uint32_t lane = threadIdx.x & 63, hk = a.kv.heads, chunks = (a.sq.count + 63) / 64;
    Start st = {};
    uint32_t x = 0, seen = 0, u = 0, incl = 0;
    // the sequences, 64 at a time, for the sum, then up to the one that holds unit x
#pragma unroll 1
    for (uint32_t it = 0; it < 2 * chunks; ++it) {
        const uint32_t s0 = 64 * (it < chunks ? it : it - chunks), s = s0 + lane;
        if (chunks > 1 || it == 0) {
            u = 0;
            if (s < a.sq.count) {
                const SeqSpan sp = seq_span(a.sq, a.kv.shift, s, a.tokens);
                u = Tiles<kRows, kUnit, kExtra>(sp.c, sp.n, a.grp).all() * hk;
            }
            incl = wave_scan(u);
        }
        const uint32_t sum = (uint32_t)__shfl((int)incl, 63);
        if (it < chunks) {
            st.total = add_units(st.total, sum);
            if (it + 1 < chunks) continue;
            if (st.total == kTooMany) return st;  // (left is 0: no workgroup has work)
            x = range_at(w, st.total, groups);
            st.left = range_at(w + 1, st.total, groups) - x;
            if (st.left == 0) return st;
            continue;
        }
        const uint64_t past = __ballot(seen + incl > x);
        if (past) {
            const int at = __ffsll((unsigned long long)past) - 1;
            st.s = s0 + (uint32_t)at;
            const uint32_t us = (uint32_t)__shfl((int)u, at), before = seen + (uint32_t)__shfl((int)incl, at) - us;
            const uint32_t per = us / hk, in = x - before;
            st.kh = in / per;
            st.unit = in % per;
            const SeqSpan sp = seq_span(a.sq, a.kv.shift, st.s, a.tokens);
            const Tiles<kRows, kUnit, kExtra> t(sp.c, sp.n, a.grp);
            // the last tile whose units begin at or before that: 64 candidates at a time
            uint32_t lo = 0, hi = t.count, first = 0;
#pragma unroll 1
            while (hi - lo > 1) {
                const uint32_t step = (hi - lo + 63) / 64, cand = lo + lane * step;
                const uint32_t b = cand < hi ? t.before(cand) : 0xffffffffu;
                const uint32_t k = (uint32_t)__popcll(__ballot(b <= st.unit)) - 1;  // (lane 0 always)
                lo += k * step;
                hi = min(hi, lo + step);
                first = (uint32_t)__shfl((int)b, (int)k);
            }
            st.tile = lo;
            st.unit -= first;
            return st;
        }
        seen += sum;
    }
    st.left = 0;  // (not reached: the range begins below the total)
    return st;
}

// Granules (8 values) of a row in LDS, permuted so that the reads below meet
// every bank once: K is read granule by granule down the rows, V in blocks of 4
// rows by 4 granules.
template <uint32_t kDim>
__device__ __forceinline__ uint32_t k_at(uint32_t row, uint32_t g) {
    constexpr uint32_t G = kDim / 8;
    return row * G + (g ^ (row & (G < 16 ? G - 1 : 15)));
}
template <uint32_t kDim>
__device__ __forceinline__ uint32_t v_at(uint32_t row, uint32_t g) {
    constexpr uint32_t G = kDim / 8;
    return row * G + (g ^ (G < 16 ? (row >> 1 & 1) * 4 : (row & 3) * 4));
}

__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Any exponent of two packed values all ones (infinities, not-a-numbers)?
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t x) {
    constexpr uint32_t e = Mma<T>::kExp * 0x10001u, one = (Mma<T>::kExp & (0u - Mma<T>::kExp)) * 0x10001u;
    return ((x & e) + one) & 0x80008000u;
}

// A weight of 0 does not hide an infinity or a not-a-number from a product, so
// a tile of V that some row does not see in full loses them here (granules
// first, first + step, ...; true if there were any); the rows that do see them
// get them back at the end, from the cache.
template <typename T>
__device__ __forceinline__ bool clean(u32x4* lv, uint32_t first, uint32_t step, uint32_t count) {
    bool found = false;
#pragma unroll 1
    for (uint32_t i = first; i < count; i += step) {
        u32x4 x = lv[i];
        if ((not_finite<T>(x[0]) | not_finite<T>(x[1]) | not_finite<T>(x[2]) | not_finite<T>(x[3])) == 0) continue;
        found = true;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t b = not_finite<T>(x[k]);
            x[k] &= (b & 0x8000u ? 0u : 0xffffu) | (b & 0x80000000u ? 0u : 0xffff0000u);
        }
        lv[i] = x;
    }
    return found;
}

// The state of a wave's 32 rows: lane l has row l % 32 (l / 32: which half of
// the keys of a block, and of the dims of a product, it holds).  A block is 32 keys.
template <typename T, uint32_t kDim>
struct WaveRows {
    typedef typename Mma<T>::V8 V8;
    static constexpr uint32_t kT = kDim / 16, kD = kDim / 32;
    static constexpr int kValu = 0x2, kMfma = 0x8, kDsRead = 0x100;  // of sched_group_barrier
    V8 q[kT];
    f32x16 o[kD];  // O^T: register i of tile d: dim 32 d + 8 (i / 4) + 4 (l / 32) + i % 4
    float m, l;    // reference of the exponents (a maximum of q . k so far); this lane's part of the sum
    uint32_t lim;  // entries that the row sees

    // Operands from LDS: 16 dims of K's rows, and 16 keys by 32 dims of V, transposed:
    // keys 16 t + 4 half + 0..3 and 16 t + 8 + 4 half + 0..3, the order that P has.
    // The first addresses of this lane in a tile of K and one of V, in bytes; the
    // order of the granules makes the others exclusive-ors of them.
    uint32_t ka, va;
    __device__ __forceinline__ void places(uint32_t lane, uint32_t k, uint32_t v) {
        const uint32_t half = lane >> 5;
        ka = k + 16 * k_at<kDim>(lane & 31, half);
        va = v + 16 * v_at<kDim>(4 * half + (lane & 15) / 4, 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + 8 * (lane & 1);
    }
    __device__ __forceinline__ V8 read_k(uint32_t at, uint32_t t) const {
        return __builtin_bit_cast(V8, *(const __attribute__((address_space(3))) u32x4*)(uintptr_t)((ka ^ (32 * t)) + at));
    }
    __device__ __forceinline__ V8 read_v(uint32_t at, uint32_t t, uint32_t d) const {
        // (8 rows on, the granules' order is the same: see v_at)
        s16x4 v[2];
#pragma unroll
        for (uint32_t w = 0; w < 2; ++w)
            v[w] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4*)(uintptr_t)((va ^ (64 * d)) + at + (16 * t + 8 * w) * 2 * kDim));
        return __builtin_bit_cast(V8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }

    __device__ __forceinline__ void read_k(V8 (&k)[kT], uint32_t at) const {
#pragma unroll
        for (uint32_t t = 0; t < kT; ++t) k[t] = read_k(at, t);
        __builtin_amdgcn_sched_barrier(0);  // (else each read is pulled down to its product, which then waits for it)
    }
    // S^T of a block: register i: key 8 (i / 4) + 4 (l / 32) + i % 4.
    __device__ __forceinline__ f32x16 scores(const V8 (&k)[kT]) const {
        f32x16 s = {};
#pragma unroll
        for (uint32_t t = 0; t < kT; ++t) s = Mma<T>::mul(k[t], q[t], s);
        return s;
    }

    // The largest of a block's scores and m (this half's).
    __device__ __forceinline__ float largest(const f32x16& s) const {
        float x = m;
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i) x = fmaxf(x, s[i]);
        return x;
    }

    // Before the step of a block from entry j0 on: the scores that the row does not see
    // go, and the sums are scaled to a new reference where the largest score asks for it.
    __device__ __forceinline__ void rescale(f32x16& s, float most, uint32_t j0, bool masked, float sl2) {
        const uint32_t half = (threadIdx.x & 63) >> 5;
        if (masked) {
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i)
                if (j0 + 8 * (i / 4) + 4 * half + i % 4 >= lim) s[i] = -INFINITY;
            most = largest(s);
        }
        const float top = max_halves(most);
        // The reference is an earlier maximum until one exceeds it by 2^8: sums and
        // weights stay far from the types' ends, and most steps scale nothing.
        if (__any((top - m) * sl2 > 8.f)) {
            // nothing but -inf so far: sums stay zero instead of inf - inf
            const float a = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - top) * sl2);
            l *= a;
#pragma unroll
            for (uint32_t d = 0; d < kD; ++d)
#pragma unroll
                for (uint32_t i = 0; i < 16; ++i) o[d][i] *= a;
            m = top;
        }
    }

    // Weights of keys 16 t .. of a block, in the cache's type, and their sum.
    __device__ __forceinline__ V8 weights(const f32x16& s, uint32_t t, float sl2, float base) {
        V8 p;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const float x = __builtin_amdgcn_exp2f(s[8 * t + i] * sl2 - base);
            l += x;
            p[i] = (T)x;
        }
        return p;
    }

    // The block's weights and its sums with V (kV: its place in the tile).  With kNext
    // also the scores of the next block from its operands k, whose products run while
    // the weights are computed, and then the operands of the block after that (`at`:
    // their place from ka on), whose reads run behind the products with V, as does the
    // search for the next scores' largest.
    template <bool kNext, uint32_t kV>
    __device__ __forceinline__ f32x16 step(const f32x16& s, V8 (&k)[kT], uint32_t at, float sl2, float& most) {
        const float base = m == -INFINITY ? 0.f : m * sl2;
        V8 p[2], v[2][kD];
        f32x16 next = {};
#pragma unroll
        for (uint32_t d = 0; d < kD; ++d) v[0][d] = read_v(kV, 0, d);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t t = 0; t < 2; ++t) p[t] = weights(s, t, sl2, base);
        if (kNext) {
            next = scores(k);
#pragma unroll
            for (uint32_t t = 0; t < kT; ++t) {
                __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kValu, 56 / kT, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t d = 0; d < kD; ++d) v[1][d] = read_v(kV, 1, d);
        __builtin_amdgcn_sched_barrier(0);
        if (kNext) read_k(k, at);
#pragma unroll
        for (uint32_t t = 0; t < 2; ++t)
#pragma unroll
            for (uint32_t d = 0; d < kD; ++d) o[d] = Mma<T>::mul(v[t][d], p[t], o[d]);
        if (kNext) {
            most = largest(next);
#pragma unroll
            for (uint32_t i = 0; i < 2 * kD; ++i) {
                __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kValu, 2, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        return next;
    }
};

template <typename T, uint32_t kDim, bool kSplit>
struct Shape {
    static constexpr uint32_t kRows = kSplit ? 32 : 128;
    static constexpr uint32_t kKeys = kSplit ? 32 : 64;              // of an LDS tile
    static constexpr uint32_t kUnit = kSplit ? 4 * kKeys : kKeys;    // keys of one unit
    static constexpr uint32_t kExtra = kSplit ? 0 : 3;
    static constexpr uint32_t kGranules = kKeys * (kDim / 8);        // of K, and of V
    static constexpr uint32_t kLoads = kGranules / 64 / (kSplit ? 1 : 4);  // of K, and of V, a wave
    // a tile a wave, or two; the waves' results take their place
    static constexpr uint32_t kTiles = (kSplit ? 4 : 2) * 2 * kGranules, kLds = kTiles > 32 * kDim ? kTiles : 32 * kDim;
    static constexpr uint32_t kPart = kRows * kDim + 2 * kRows;      // floats of a part
};

// 16 zero bytes: what lanes beyond the head's dim load.
__device__ const u32x4 kZeroGranule = {0, 0, 0, 0};

// 16 bytes a lane from global memory to LDS at byte `to` (the wave's) + 16 lane,
// from an address a lane, or from a base that the wave shares and an offset a
// lane.  By hand: with the builtin every later LDS read waits for all loads in
// flight, which ends the overlap.  The compiler does not count these loads;
// wait_loads comes before their data is read.
__device__ __forceinline__ void load_lds(const void* from, uint32_t to) {
    uint32_t saved;  // (the compiler may hold something in m0, which cannot be named as clobbered)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved)
                 : "v"(from), "s"(uniform(to))
                 : "memory");
}
__device__ __forceinline__ uint64_t uniform(const void* p) {
    const uint64_t x = (uint64_t)p;
    return (uint64_t)uniform((uint32_t)(x >> 32)) << 32 | uniform((uint32_t)x);
}
// Two loads, to `to` and 1024 bytes on (in one statement, so that m0 is saved once).
__device__ __forceinline__ void load_lds(const void* base0, uint32_t offset0, const void* base1, uint32_t offset1, uint32_t to) {
    uint32_t saved;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %5\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\t"
                 "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %4\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved)
                 : "v"(offset0), "s"(uniform(base0)), "v"(offset1), "s"(uniform(base1)), "s"(uniform(to))
                 : "memory", "scc");
}
// All but the kNewest last loads of this wave have landed.  (The builtin, unlike
// assembly, tells the compiler that its own loads have: it would wait for them
// again inside the loops, and with them for the loads in flight.)
template <uint32_t kNewest>
__device__ __forceinline__ void wait_loads() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((kNewest & 15) | 7 << 4 | 15 << 8 | (kNewest >> 4) << 14);
    asm volatile("" ::: "memory");
}
// The LDS reads of this wave are done: their place may be filled again.
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Parts are written and read past the L2s, which do not see each other's lines.
__device__ __forceinline__ void put_part(float* p, float x, float y) {
    const u32x2 v = {__float_as_uint(x), __float_as_uint(y)};
    __hip_atomic_store((uint64_t*)p, __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get_part(const float* p) {
    const u32x2 v = __builtin_bit_cast(
        u32x2, __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    return {__uint_as_float(v[0]), __uint_as_float(v[1])};
}

// Four consecutive values of a row of the output.
__device__ __forceinline__ void put4(const TileArgs& a, size_t at, f32x4 x) {
    typedef __bf16 B4 __attribute__((ext_vector_type(4)));
    typedef _Float16 H4 __attribute__((ext_vector_type(4)));
    if (!a.wide_out) {
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
            const float y = i == 0 ? x[0] : i == 1 ? x[1] : i == 2 ? x[2] : x[3];
            store_as(a.out.p, a.out.type, at + i, y, a.inv_scale);
        }
    } else if (a.out.type == MVK_TYPE_BF16) {
        *(u32x2*)((uint16_t*)a.out.p + at) = __builtin_bit_cast(u32x2, __builtin_convertvector(x, B4));
    } else if (a.out.type == MVK_TYPE_F16) {
        *(u32x2*)((uint16_t*)a.out.p + at) = __builtin_bit_cast(u32x2, __builtin_convertvector(x, H4));
    } else if (a.out.type == MVK_TYPE_F32) {
        *(f32x4*)((float*)a.out.p + at) = x;
    } else {
        *(u32x4*)((uint32_t*)a.out.p + at) = u32x4{field_of(x[0] * a.inv_scale), field_of(x[1] * a.inv_scale),
                                                   field_of(x[2] * a.inv_scale), field_of(x[3] * a.inv_scale)};
    }
}

// A lane's part of its row, dims 8 i .. 8 i + 3 from `at` on (aligned outputs); one
// loop a type, so that the type is not asked for at every store.
template <uint32_t kDim>
__device__ __forceinline__ void put_rows(const TileArgs& a, size_t at, const f32x16* o, float f) {
    typedef __bf16 B4 __attribute__((ext_vector_type(4)));
    typedef _Float16 H4 __attribute__((ext_vector_type(4)));
    const uint32_t live = a.kv.dim / 8;
    auto value = [&](uint32_t i) {
        const f32x16& x = o[i / 4];
        return f32x4{x[4 * (i % 4)], x[4 * (i % 4) + 1], x[4 * (i % 4) + 2], x[4 * (i % 4) + 3]} * f;
    };
    if (a.out.type == MVK_TYPE_BF16) {
#pragma unroll
        for (uint32_t i = 0; i < kDim / 8; ++i)
            if (i < live) *(u32x2*)((uint16_t*)a.out.p + at + 8 * i) = __builtin_bit_cast(u32x2, __builtin_convertvector(value(i), B4));
    } else if (a.out.type == MVK_TYPE_F16) {
#pragma unroll
        for (uint32_t i = 0; i < kDim / 8; ++i)
            if (i < live) *(u32x2*)((uint16_t*)a.out.p + at + 8 * i) = __builtin_bit_cast(u32x2, __builtin_convertvector(value(i), H4));
    } else {
        const bool field = a.out.type == MVK_TYPE_FIELD;
#pragma unroll
        for (uint32_t i = 0; i < kDim / 8; ++i)
            if (i < live) {
                f32x4 x = value(i);
                if (field) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[k] = __uint_as_float(field_of(x[k] * a.inv_scale));
                }
                *(f32x4*)((float*)a.out.p + at + 8 * i) = x;
            }
    }
}

__device__ __forceinline__ void put_lse(const TileArgs& a, size_t at, float m, float l) {
    a.lse[at] = l > 0.f ? (m * a.sl2 + __builtin_log2f(l)) * kLn2 : l == 0.f ? -INFINITY : l;
}

// Four values y (not yet divided by the sum l) of row `row` of (sequence, kv head), dims 4 g and on.
__device__ __forceinline__ void put_row(const TileArgs& a, const SeqSpan& sp, uint32_t kh, uint32_t row, uint32_t g,
                                        f32x4 y, float m, float l) {
    const uint32_t t = sp.q0 + row / a.grp, h = kh * a.grp + row % a.grp;
    // (a sum that is not a number stays one; a row without entries is zero, its sums are)
    put4(a, (size_t)t * a.out.token + (size_t)h * a.out.head + 4 * g, y * (l > 0.f ? 1.f / l : l));
    if (a.lse && g == 0) put_lse(a, (size_t)t * a.heads + h, m, l);
}

constexpr uint32_t kCounterStride = 16;

// C: how the cache holds its values (T itself, or in 8 bits).
template <typename T, typename C, uint32_t kDim, bool kSplit>
__global__ __launch_bounds__(256, kDim > 128 ? 1 : 2) void attend_tile(TileArgs a) {
    typedef Shape<T, kDim, kSplit> Sh;
    typedef typename Mma<T>::V8 V8;
    typedef typename Held<C>::S S;
    constexpr bool k8 = Held<C>::k8;
    constexpr uint32_t G = kDim / 8;  // granules a row
    __shared__ __attribute__((aligned(65536))) u32x4 lds[Sh::kLds];  // (at 0: see kTile)
    __shared__ float red[4][32][2];
    __shared__ uint32_t last_one, cleaned[2];  // (cleaned: of this segment and the next)
    const uint32_t tid = threadIdx.x, wave = uniform(tid >> 6);
    const uint32_t dim = a.kv.dim, live = dim / 8;  // granules of a row that hold data
    // consecutive ranges on one XCD, whose L2 then holds the keys they share
    const uint32_t groups = gridDim.x, xcds = groups % 8 == 0 ? 8 : 1;
    const uint32_t w = (blockIdx.x % xcds) * (groups / xcds) + blockIdx.x / xcds;
    Start st = find_start<Sh::kRows, Sh::kUnit, Sh::kExtra>(a, w, groups);
    st = {uniform(st.s), uniform(st.kh), uniform(st.tile), uniform(st.unit), uniform(st.left), uniform(st.total)};
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
    u32x4* const mine = kSplit ? lds + wave * 2 * Sh::kGranules : lds;
    // load i of this wave fills 64 granules from granule 64 (i + kLoads wave) of the tile on
    const uint32_t part0 = kSplit ? 0 : 64 * Sh::kLoads * wave;

    if (tid < 2) cleaned[tid] = 0;
    __syncthreads();
    uint32_t done = 0, turn = 0;
    SeqSpan sp = {};
    uint32_t ids = 0, id0 = 0, id1 = 0;  // lane i: the page of the sequence's pages id0 + i, of id0 .. id1 - 1
    auto sequence = [&]() {
        const SeqSpan x = seq_span(a.sq, a.kv.shift, st.s, a.tokens);
        sp = {uniform(x.q0), uniform(x.c), uniform(x.n)};
        id0 = id1 = 0;
    };
    if (st.left) sequence();
#pragma unroll 1
    while (done < st.left) {
        // (unknown to the compiler, which would otherwise keep every address of the
        // beginnings and ends of tiles in registers that the loops need)
        uint32_t lane = tid & 63;
        asm volatile("" : "+v"(lane));
        const uint32_t col = lane & 31, half = lane >> 5;
        const Tiles<Sh::kRows, Sh::kUnit, Sh::kExtra> tiles(sp.c, sp.n, a.grp);
        const uint32_t units = tiles.units(st.tile);
        const uint32_t u0 = st.unit, u1 = min(units, u0 + (st.left - done));

        // rows
        const uint32_t rows = sp.c * a.grp, tile0 = st.tile * Sh::kRows, row0 = tile0 + (kSplit ? 0 : 32 * wave);
        const uint32_t known = min(row0 + col, rows - 1);
        // keys
        const char* const kb = (const char*)((const S*)a.kv.K + (size_t)st.kh * a.kv.kh);
        const char* const vb = (const char*)((const S*)a.kv.V + (size_t)st.kh * a.kv.vh);
        const uint32_t mask = (1u << a.kv.shift) - 1;
        const uint32_t key0 = (max(u0, Sh::kExtra) - Sh::kExtra) * Sh::kUnit, key1 = (max(u1, Sh::kExtra) - Sh::kExtra) * Sh::kUnit;
        const uint32_t first = key0 + (kSplit ? wave * Sh::kKeys : 0);
        const uint32_t stop = min(key1, sp.n);  // entries at and beyond it are not needed
        // before the loads of the tile at j0: its pages are known (places beyond the
        // last page in use are read in that page, so no address leaves the pool)
        auto pages = [&](uint32_t j0) {
            if ((min(j0 + Sh::kKeys, sp.n) - 1) >> a.kv.shift >= id1 || j0 >> a.kv.shift < id0) {
                id0 = j0 >> a.kv.shift;
                id1 = id0 + 64;
                ids = seq_page(a.sq, a.kv, st.s, min((id0 + lane) << a.kv.shift, sp.n - 1));
            }
        };
        // load i of the wave: granules part0 + 64 i + lane of the tile, that is rows kStep i + lane / G on
        constexpr uint32_t kStep = 64 / G > 0 ? 64 / G : 1;
        const uint32_t lane_row = part0 / G + lane / G;
        auto granule = [&](bool is_v, uint32_t r) { return (is_v ? v_at<kDim>(r, lane % G) : k_at<kDim>(r, lane % G)) % G; };
        auto load = [&](const char* base, size_t page_stride, size_t entry_stride, bool is_v, uint32_t j0, uint32_t to) {
            if (a.whole_page) {
                // a base that the wave shares, and 32-bit offsets of which a few differ
                const uint32_t pg = (uint32_t)__builtin_amdgcn_readlane((int)ids, (int)((j0 >> a.kv.shift) - id0));
                const char* b = base + ((size_t)pg * page_stride + (size_t)(j0 & mask) * entry_stride) * sizeof(T);
                auto from = [&](uint32_t i) { return b + (size_t)(kStep * i * (uint32_t)entry_stride * sizeof(T)); };
                auto offset = [&](uint32_t i) {
                    return (uint32_t)((lane_row * (uint32_t)entry_stride + 8 * granule(is_v, kStep * i + lane_row)) * sizeof(T));
                };
                static_assert(Sh::kLoads % 2 == 0, "two at a time");
#pragma unroll
                for (uint32_t i = 0; i < Sh::kLoads; i += 2) load_lds(from(i), offset(i), from(i + 1), offset(i + 1), to + 1024 * i);
            } else {
                const uint32_t used = (sp.n - 1) >> a.kv.shift;
#pragma unroll 1
                for (uint32_t i = 0; i < Sh::kLoads; ++i) {
                    const uint32_t r = kStep * i + lane_row, g = granule(is_v, r), j = j0 + r;
                    const size_t pg = (uint32_t)__shfl((int)ids, (int)(min(j >> a.kv.shift, used) - id0));
                    const void* from = base + (pg * page_stride + (size_t)(j & mask) * entry_stride + 8 * g) * sizeof(T);
                    load_lds(g < live ? from : (const void*)&kZeroGranule, to + 1024 * i);
                }
            }
        };
        auto load_k = [&](uint32_t j0, uint32_t stage) {
            load(kb, a.kv.kp, a.kv.ke, false, j0, lds0 + 16 * ((kSplit ? wave : stage) * 2 * Sh::kGranules + part0));
        };
        auto load_v = [&](uint32_t j0, uint32_t stage) {
            load(vb, a.kv.vp, a.kv.ve, true, j0, lds0 + 16 * ((kSplit ? wave : stage) * 2 * Sh::kGranules + Sh::kGranules + part0));
        };
        // A cache held in 8 bits: this wave's granules of a tile go by way of registers, where
        // they are widened.  An exponent a row; lane i has that of the wave's row i.
        constexpr uint32_t kMine = 64 * Sh::kLoads / G;  // rows
        struct Codes {
            u32x2 c[k8 ? Sh::kLoads : 1];
            int e;
        };
        // (the lane is unknown to the compiler in each: it would keep all their addresses in
        // registers that the loops need)
        auto fetch = [&](bool is_v, uint32_t j0, Codes& to) {
            uint32_t ln = lane;
            asm volatile("" : "+v"(ln));
            const uint32_t first_row = part0 / G + ln / G;
            auto granule_of = [&](uint32_t r) { return (is_v ? v_at<kDim>(r, ln % G) : k_at<kDim>(r, ln % G)) % G; };
            const char* base = is_v ? vb : kb;
            const size_t page_stride = is_v ? a.kv.vp : a.kv.kp, entry_stride = is_v ? a.kv.ve : a.kv.ke;
            const int8_t* ex = is_v ? a.kv.vx + (size_t)st.kh * a.kv.vxh : a.kv.kx + (size_t)st.kh * a.kv.kxh;
            const size_t xp = is_v ? a.kv.vxp : a.kv.kxp, xe = is_v ? a.kv.vxe : a.kv.kxe;
            const uint32_t row = part0 / G + ln % kMine;
            if (a.whole_page) {
                const uint32_t pg = (uint32_t)__builtin_amdgcn_readlane((int)ids, (int)((j0 >> a.kv.shift) - id0));
                const char* b = base + (size_t)pg * page_stride + (size_t)(j0 & mask) * entry_stride;
#pragma unroll
                for (uint32_t i = 0; i < Sh::kLoads; ++i)
                    to.c[k8 ? i : 0] = *(const u32x2*)(b + (first_row * (uint32_t)entry_stride + 8 * granule_of(kStep * i + first_row)) +
                                              (size_t)(kStep * i * (uint32_t)entry_stride));
                to.e = ex[(size_t)pg * xp + (size_t)(j0 & mask) * xe + row * (uint32_t)xe];
            } else {
                const uint32_t used = (sp.n - 1) >> a.kv.shift;
#pragma unroll
                for (uint32_t i = 0; i < Sh::kLoads; ++i) {
                    const uint32_t r = kStep * i + first_row, g = granule_of(r), j = j0 + r;
                    const size_t pg = (uint32_t)__shfl((int)ids, (int)(min(j >> a.kv.shift, used) - id0));
                    const char* from = base + pg * page_stride + (size_t)(j & mask) * entry_stride + 8 * g;
                    to.c[k8 ? i : 0] = *(const u32x2*)(g < live ? from : (const char*)&kZeroGranule);
                }
                const uint32_t j = j0 + row;
                const size_t pg = (uint32_t)__shfl((int)ids, (int)(min(j >> a.kv.shift, used) - id0));
                to.e = ex[pg * xp + (size_t)(j & mask) * xe];
            }
            __builtin_amdgcn_sched_barrier(0);  // (all asked for here, not where they are used)
        };
        auto put = [&](bool is_v, const Codes& from, uint32_t stage) {
            uint32_t ln = lane;
            asm volatile("" : "+v"(ln));
            u32x4* const to = lds + (kSplit ? wave : stage) * 2 * Sh::kGranules + (is_v ? Sh::kGranules : 0) + part0 + ln;
            const float two = power(from.e);
#pragma unroll
            for (uint32_t i = 0; i < Sh::kLoads; ++i) {
                const float f = __shfl(two, (int)((kStep * i + ln / G) % kMine));
                to[64 * i] = __builtin_bit_cast(u32x4, widen<C>(from.c[k8 ? i : 0], f));
            }
            asm volatile("" ::: "memory");
        };
        Codes ck, cv;
        // The chunks form has no registers for that while it computes: the codes go to LDS as they
        // are, 16 a lane, into this wave's part of the place that they are widened in later.
        constexpr uint32_t kRaw = k8 && !kSplit ? kDim / 64 : 1, kLanes = kDim / 16;  // loads a wave; lanes a row
        struct Exps {
            int e[kRaw];
        };
        auto place8 = [&](bool is_v, uint32_t stage) { return (stage * 2 + (is_v ? 1 : 0)) * Sh::kGranules + part0; };
        auto fetch_raw = [&](bool is_v, uint32_t j0, uint32_t stage, Exps& to) {
            uint32_t ln = lane;
            asm volatile("" : "+v"(ln));
            const uint32_t raw_row = part0 / G + ln / kLanes, raw_at = ln % kLanes * 16;
            const char* base = is_v ? vb : kb;
            const size_t page_stride = is_v ? a.kv.vp : a.kv.kp, entry_stride = is_v ? a.kv.ve : a.kv.ke;
            const int8_t* ex = is_v ? a.kv.vx + (size_t)st.kh * a.kv.vxh : a.kv.kx + (size_t)st.kh * a.kv.kxh;
            const size_t xp = is_v ? a.kv.vxp : a.kv.kxp, xe = is_v ? a.kv.vxe : a.kv.kxe;
            const uint32_t used = (sp.n - 1) >> a.kv.shift;
#pragma unroll
            for (uint32_t i = 0; i < kRaw; ++i) {
                const uint32_t r = raw_row + 64 / kLanes * i, j = j0 + r;
                const size_t pg = (uint32_t)__shfl((int)ids, (int)(min(j >> a.kv.shift, used) - id0));
                const char* from = base + pg * page_stride + (size_t)(j & mask) * entry_stride + raw_at;
                load_lds(raw_at < dim ? from : (const char*)&kZeroGranule, lds0 + 16 * (place8(is_v, stage) + 64 * i));
                to.e[i] = ex[pg * xp + (size_t)(j & mask) * xe];
            }
        };
        // (its reads come before its writes, in this wave's order; no other wave uses the part)
        auto widen_raw = [&](bool is_v, uint32_t stage, const Exps& from) {
            uint32_t ln = lane;
            asm volatile("" : "+v"(ln));
            const uint32_t raw_row = part0 / G + ln / kLanes, raw_at = ln % kLanes * 16;
            u32x4* const tile = lds + (stage * 2 + (is_v ? 1 : 0)) * Sh::kGranules;
            u32x4 c[kRaw];
#pragma unroll
            for (uint32_t i = 0; i < kRaw; ++i) c[i] = lds[place8(is_v, stage) + 64 * i + ln];
            asm volatile("" ::: "memory");
#pragma unroll
            for (uint32_t i = 0; i < kRaw; ++i) {
                const uint32_t r = raw_row + 64 / kLanes * i;
                const float two = power(from.e[i]);
#pragma unroll
                for (uint32_t h = 0; h < 2; ++h) {
                    const uint32_t g = raw_at / 8 + h;
                    tile[is_v ? v_at<kDim>(r, g) : k_at<kDim>(r, g)] =
                        __builtin_bit_cast(u32x4, widen<C>(u32x2{c[i][2 * h], c[i][2 * h + 1]}, two));
                }
            }
            asm volatile("" ::: "memory");
        };
        // The tokens form takes K from memory to the operands' registers: a lane has a key, half of
        // its dims, 16 at a time (so product t has dims 32 (t / 2) + 16 half + 8 (t % 2) and on, of q too).
        struct KeyCodes {
            u32x4 c[k8 && kSplit ? kDim / 32 : 1];
            int e;
        };
        auto fetch_key = [&](uint32_t j0, KeyCodes& to) {
            uint32_t ln = lane;
            asm volatile("" : "+v"(ln));
            const uint32_t j = j0 + (ln & 31), at = 16 * (ln >> 5);
            const size_t pg = (uint32_t)__shfl((int)ids, (int)((min(j, sp.n - 1) >> a.kv.shift) - id0));
            const char* from = kb + pg * a.kv.kp + (size_t)(j & mask) * a.kv.ke + at;
            if (a.by_16) {
#pragma unroll
                for (uint32_t i = 0; i < kDim / 32; ++i)
                    to.c[k8 && kSplit ? i : 0] = *(const u32x4*)(32 * i + at < dim ? from + 32 * i : (const char*)&kZeroGranule);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < kDim / 32; ++i) {
                    const u32x2 x = *(const u32x2*)(32 * i + at < dim ? from + 32 * i : (const char*)&kZeroGranule);
                    const u32x2 y = *(const u32x2*)(32 * i + at + 8 < dim ? from + 32 * i + 8 : (const char*)&kZeroGranule);
                    to.c[k8 && kSplit ? i : 0] = u32x4{x[0], x[1], y[0], y[1]};
                }
            }
            to.e = a.kv.kx[(size_t)st.kh * a.kv.kxh + pg * a.kv.kxp + (size_t)(j & mask) * a.kv.kxe];
            __builtin_amdgcn_sched_barrier(0);
        };
        KeyCodes kk;
        // the first loads of keys, then the rows, which arrive behind them
        if (k8) {
            if (first < stop) {
                pages(first);
                if (kSplit) {
                    fetch_key(first, kk);
                    fetch(true, first, cv);
                } else {
                    fetch(false, first, ck);
                }
            }
        } else if (first < stop) {
            pages(first);
            load_k(first, 0);
            load_v(first, 0);
            if (!kSplit && first + Sh::kUnit < stop) {
                pages(first + Sh::kUnit);
                load_k(first + Sh::kUnit, 1);
            }
        }

        WaveRows<T, kDim> x;
        {
            const uint32_t tok = known / a.grp, head = st.kh * a.grp + known % a.grp;
            const int64_t see = (int64_t)sp.n - sp.c + tok + 1;
            x.lim = see > 0 ? (uint32_t)see : 0u;
            const T* qr = (const T*)a.q.p + (size_t)(sp.q0 + tok) * a.q.token + (size_t)head * a.q.head;
            u32x4 v[kDim / 16];  // (rows and granules that are not there: zeros, so that all loads are in flight at once)
#pragma unroll
            for (uint32_t t = 0; t < kDim / 16; ++t) {
                const uint32_t g = k8 && kSplit ? 4 * (t / 2) + 2 * half + t % 2 : 2 * t + half;
                v[t] = *(row0 + col < rows && g < live ? (const u32x4*)(qr + 8 * g) : &kZeroGranule);
            }
#pragma unroll
            for (uint32_t t = 0; t < kDim / 16; ++t) x.q[t] = __builtin_bit_cast(V8, v[t] ^ a.flip);
#pragma unroll
            for (uint32_t d = 0; d < kDim / 32; ++d) x.o[d] = f32x16{};
            x.m = -INFINITY;
            x.l = 0.f;
        }
        // limits of the wave's rows: rows are in order, so lane 0 sees least
        const uint32_t lim_lo = uniform(x.lim);
        const uint32_t lim_hi = (uint32_t)__builtin_amdgcn_readlane((int)x.lim, 31);
        const uint32_t lim_0 = (uint32_t)max((int64_t)sp.n - sp.c + tile0 / a.grp + 1, (int64_t)0);  // of the tile's rows
        const bool idle = !kSplit && row0 >= rows;  // a wave without rows

        x.places(lane, lds0 + (kSplit ? wave * 32 * Sh::kGranules : 0), lds0 + (kSplit ? wave * 32 * Sh::kGranules : 0) + 16 * Sh::kGranules);
        if (kSplit && k8) {
            // (a wave's writes and reads of LDS are in its own order)
#pragma unroll 1
            for (uint32_t j0 = first; j0 < stop; j0 += Sh::kUnit) {
                const bool more = j0 + Sh::kUnit < stop, masked = j0 + Sh::kKeys > lim_lo;
                V8 k[kDim / 16];
                const float two = power(kk.e);
#pragma unroll
                for (uint32_t t = 0; t < kDim / 16; ++t) {
                    const u32x4 c = kk.c[k8 && kSplit ? t / 2 : 0];
                    k[t] = __builtin_bit_cast(V8, widen<C>(u32x2{c[2 * (t % 2)], c[2 * (t % 2) + 1]}, two));
                }
                if (more) {
                    pages(j0 + Sh::kUnit);
                    fetch_key(j0 + Sh::kUnit, kk);
                }
                f32x16 s = x.scores(k);
                float most = x.largest(s);
                x.rescale(s, most, j0, masked, a.sl2);
                put(true, cv, 0);
                if (more) fetch(true, j0 + Sh::kUnit, cv);
                if (masked && __any(clean<T>(mine + Sh::kGranules, lane, 64, Sh::kGranules))) cleaned[turn] = 1;
                x.template step<false, 0>(s, k, 0, a.sl2, most);
            }
        } else if (kSplit) {
#pragma unroll 1
            for (uint32_t j0 = first; j0 < stop; j0 += Sh::kUnit) {
                const bool more = j0 + Sh::kUnit < stop, masked = j0 + Sh::kKeys > lim_lo;
                wait_loads<Sh::kLoads>();  // K
                V8 k[kDim / 16];
                x.read_k(k, 0);
                f32x16 s = x.scores(k);
                if (more) {
                    pages(j0 + Sh::kUnit);
                    wait_reads();
                    load_k(j0 + Sh::kUnit, 0);
                }
                float most = x.largest(s);
                x.rescale(s, most, j0, masked, a.sl2);
                if (more) wait_loads<Sh::kLoads>();
                else wait_loads<0>();
                if (masked && __any(clean<T>(mine + Sh::kGranules, lane, 64, Sh::kGranules))) cleaned[turn] = 1;
                x.template step<false, 0>(s, k, 0, a.sl2, most);
                wait_reads();
                if (more) load_v(j0 + Sh::kUnit, 0);
            }
        } else if (first < stop) {
            // Two blocks a tile.  The scores of a block are formed during the step before
            // it, from operands read during the step before that; so when a tile's steps
            // begin, its K has been read, and the next tile's K and its V are there.
            const uint32_t end = idle ? 0 : min(stop, lim_hi);  // blocks from here on say nothing to this wave
            constexpr uint32_t kTile = 32 * Sh::kGranules, kBlock = 8 * Sh::kGranules;  // bytes
            static_assert((kTile & (kTile - 1)) == 0, "one bit tells the tiles apart");
            uint32_t stage = 0;
            if (k8) {
                put(false, ck, 0);
                fetch(true, first, ck);
                put(true, ck, 0);
                if (first + Sh::kUnit < stop) {
                    pages(first + Sh::kUnit);
                    fetch(false, first + Sh::kUnit, ck);
                    put(false, ck, 1);
                }
            } else {
                wait_loads<0>();
            }
            __syncthreads();
            f32x16 s0 = {}, s1 = {};
            V8 k[kDim / 16];
            x.read_k(k, 0);
            float most = 0.f;
            if (first < end) {
                s0 = x.scores(k);
                most = x.largest(s0);
            }
            x.read_k(k, kBlock);
#pragma unroll 1
            for (uint32_t j0 = first; j0 < stop; j0 += Sh::kUnit) {
                if (!k8) wait_loads<0>();
                __syncthreads();
                const bool next_v = j0 + Sh::kUnit < stop, next_k = j0 + 2 * Sh::kUnit < stop;
                Exps ke, ve;
                if (k8) {
                    if (a.by_16) {
                        if (next_v) fetch_raw(true, j0 + Sh::kUnit, stage ^ 1, ve);
                        if (next_k) {
                            pages(j0 + 2 * Sh::kUnit);
                            fetch_raw(false, j0 + 2 * Sh::kUnit, stage, ke);
                        }
                    }
                } else {
                    if (next_v) load_v(j0 + Sh::kUnit, stage ^ 1);
                    if (next_k) {
                        pages(j0 + 2 * Sh::kUnit);
                        load_k(j0 + 2 * Sh::kUnit, stage);
                    }
                }
                if (j0 + Sh::kKeys > lim_0) {  // for all waves alike
                    if (clean<T>(mine + (2 * stage + 1) * Sh::kGranules, tid, 256, Sh::kGranules)) cleaned[turn] = 1;
                    __syncthreads();
                }
                stage ^= 1;
                x.ka ^= kTile;
                if (j0 < end) {
                    x.rescale(s0, most, j0, j0 + 32 > lim_lo, a.sl2);
                    // the wave with products to issue goes first: the two workgroups of a
                    // compute unit then take turns (chunk of 512 over 16000: 2 % faster)
                    __builtin_amdgcn_s_setprio(1);
                    s1 = x.template step<true, 0>(s0, k, 0, a.sl2, most);
                    __builtin_amdgcn_s_setprio(0);
                }
                if (j0 + 32 < end) {
                    x.rescale(s1, most, j0 + 32, j0 + 64 > lim_lo, a.sl2);
                    __builtin_amdgcn_s_setprio(1);
                    s0 = x.template step<true, kBlock>(s1, k, kBlock, a.sl2, most);
                    __builtin_amdgcn_s_setprio(0);
                }
                x.va ^= kTile;
                if (k8 && a.by_16) {  // (stage is the next tile's by now; the K that was in the other has been read)
                    wait_loads<0>();
                    if (next_v) widen_raw(true, stage, ve);
                    if (next_k) widen_raw(false, stage ^ 1, ke);
                } else if (k8) {
                    if (next_v) {
                        fetch(true, j0 + Sh::kUnit, ck);
                        put(true, ck, stage);
                    }
                    if (next_k) {
                        pages(j0 + 2 * Sh::kUnit);
                        fetch(false, j0 + 2 * Sh::kUnit, ck);
                        put(false, ck, stage ^ 1);
                    }
                }
            }
        }

        // The results.  Infinities and not-a-numbers that a row sees in the tiles that
        // lost theirs come back first (key by key; rare).
        __syncthreads();
        const bool whole = u0 == 0 && u1 == units;
        if (uniform(cleaned[turn])) {
            const uint32_t fix0 = max(lim_0 / Sh::kKeys * Sh::kKeys, key0);
            const bool mine_first = !kSplit || wave == 0;  // (the waves of the tokens form are added)
#pragma unroll 1
            for (uint32_t j = fix0; j < stop; ++j) {
                const size_t pg = seq_page(a.sq, a.kv, st.s, j);
                const S* v = (const S*)vb + pg * a.kv.vp + (j & mask) * a.kv.ve;
                const float two = k8 ? power(a.kv.vx[pg * a.kv.vxp + (size_t)st.kh * a.kv.vxh + (j & mask) * a.kv.vxe]) : 1.f;
#pragma unroll
                for (uint32_t i = 0; i < kDim / 8; ++i) {
                    typedef S T4 __attribute__((ext_vector_type(4)));
                    if (i >= live || j >= x.lim || !mine_first) continue;
                    const T4 f = *(const T4*)(v + 8 * i + 4 * half);
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) {
                        const float y = Held<C>::get(f[k], two);
                        if (y - y != 0.f) x.o[i / 4][4 * (i % 4) + k] += y;
                    }
                }
            }
        }
        if (tid == 0) cleaned[turn ^ 1] = 0;  // (last read before the barrier that ended the segment before)
        float* const part = a.part + (size_t)(2 * w + (u0 == 0 ? 1 : 0)) * Sh::kPart;
        // the tile's ranges w0 .. w1 where there are several; counted on the first one's word
        uint32_t w0 = 0, w1 = 0;
        if (!whole) {
            const uint32_t at = range_at(w, st.total, groups) + done - u0;
            w0 = range_of(at, st.total, groups), w1 = range_of(at + units - 1, st.total, groups);
        }
        // After this workgroup's part is written: is it the last of the tile's?
        auto last_of_tile = [&]() {
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
            if (tid == 0) {
                uint32_t* c = a.counters + w0 * kCounterStride;
                const bool is_last = atomicAdd(c, 1u) == w1 - w0;
                if (is_last) atomicExch(c, 0u);
                last_one = is_last;
            }
            __syncthreads();
            return uniform(last_one) != 0;
        };
        float l = sum_halves(x.l);
        if (!kSplit) {
            // each wave its own rows, from registers: four values a lane, lane after lane
            constexpr uint32_t kSums = 32 * kDim;  // floats of a wave's sums
            bool out = true;
            if (!whole) {
                float* p = part + wave * kSums + 4 * lane;
#pragma unroll
                for (uint32_t i = 0; i < kDim / 8; ++i) {
                    put_part(p + 256 * i, x.o[i / 4][4 * (i % 4)], x.o[i / 4][4 * (i % 4) + 1]);
                    put_part(p + 256 * i + 2, x.o[i / 4][4 * (i % 4) + 2], x.o[i / 4][4 * (i % 4) + 3]);
                }
                if (half == 0) put_part(part + 4 * kSums + 64 * wave + 2 * col, x.m, l);
                out = last_of_tile();
                if (out) {
                    x.m = -INFINITY, l = 0.f;
#pragma unroll
                    for (uint32_t d = 0; d < kDim / 32; ++d) x.o[d] = f32x16{};
                    // two parts' loads in flight
#pragma unroll 1
                    for (uint32_t v = w0; v <= w1; v += 2) {
                        float2 ml[2], y[2][kDim / 4];
#pragma unroll
                        for (uint32_t u = 0; u < 2; ++u) {
                            const uint32_t vu = min(v + u, w1);
                            const float* from = a.part + (size_t)(2 * vu + (vu == w0 ? 1 : 0)) * Sh::kPart;
                            ml[u] = get_part(from + 4 * kSums + 64 * wave + 2 * col);
#pragma unroll
                            for (uint32_t i = 0; i < kDim / 4; ++i)
                                y[u][i] = get_part(from + wave * kSums + 4 * lane + 256 * (i / 2) + 2 * (i % 2));
                        }
#pragma unroll
                        for (uint32_t u = 0; u < 2; ++u) {
                            if (v + u > w1) break;
                            const float top = fmaxf(x.m, ml[u].x), base = top == -INFINITY ? 0.f : top * a.sl2;
                            const float fa = __builtin_amdgcn_exp2f(x.m * a.sl2 - base), fb = __builtin_amdgcn_exp2f(ml[u].x * a.sl2 - base);
                            x.m = top;
                            l = l * fa + ml[u].y * fb;
#pragma unroll
                            for (uint32_t i = 0; i < kDim / 4; ++i) {
                                x.o[i / 8][2 * (i % 8)] = x.o[i / 8][2 * (i % 8)] * fa + y[u][i].x * fb;
                                x.o[i / 8][2 * (i % 8) + 1] = x.o[i / 8][2 * (i % 8) + 1] * fa + y[u][i].y * fb;
                            }
                        }
                    }
                }
            }
            if (out && a.wide_out) {
                if (row0 + col < rows) {
                    const uint32_t tok = known / a.grp, head = st.kh * a.grp + known % a.grp;
                    const float inv = l > 0.f ? 1.f / l : l;  // (zero for a row without entries; its sums are zeros)
                    put_rows<kDim>(a, (size_t)(sp.q0 + tok) * a.out.token + (size_t)head * a.out.head + 4 * half, x.o, inv);
                    if (a.lse && half == 0) put_lse(a, (size_t)(sp.q0 + tok) * a.heads + head, x.m, l);
                }
                out = false;
            }
            if (out) {
                // rows without alignment: by way of LDS, value by value
                float* const all = (float*)lds + wave * kSums;
#pragma unroll
                for (uint32_t i = 0; i < kDim / 8; ++i)
                    *(f32x4*)(all + col * kDim + ((2 * i + half) ^ (col & 7)) * 4) =
                        f32x4{x.o[i / 4][4 * (i % 4)], x.o[i / 4][4 * (i % 4) + 1], x.o[i / 4][4 * (i % 4) + 2], x.o[i / 4][4 * (i % 4) + 3]};
                if (half == 0) red[wave][col][0] = x.m, red[wave][col][1] = l;
                wait_reads();
#pragma unroll 1
                for (uint32_t i = lane; i < 32 * (kDim / 4); i += 64) {
                    const uint32_t r = i / (kDim / 4), g = i % (kDim / 4);
                    if (4 * g < dim && row0 + r < rows)
                        put_row(a, sp, st.kh, row0 + r, g, *(const f32x4*)(all + r * kDim + (g ^ (r & 7)) * 4), red[wave][r][0], red[wave][r][1]);
                }
            }
        } else {
            // the waves' sums by way of LDS: wave, row, dim, four dims a granule, permuted like the keys
            float* const all = (float*)lds;
            if (half == 0) red[wave][col][0] = x.m, red[wave][col][1] = l;
#pragma unroll
            for (uint32_t i = 0; i < kDim / 8; ++i)
                *(f32x4*)(all + (wave * 32 + col) * kDim + ((2 * i + half) ^ (col & 7)) * 4) =
                    f32x4{x.o[i / 4][4 * (i % 4)], x.o[i / 4][4 * (i % 4) + 1], x.o[i / 4][4 * (i % 4) + 2], x.o[i / 4][4 * (i % 4) + 3]};
            __syncthreads();
            const uint32_t count = min(rows - tile0, Sh::kRows);
#pragma unroll 1
            for (uint32_t i = tid; i < count * (kDim / 4); i += 256) {
                const uint32_t r = i / (kDim / 4), g = i % (kDim / 4);
                if (4 * g >= dim) continue;
                const float m = fmaxf(fmaxf(red[0][r][0], red[1][r][0]), fmaxf(red[2][r][0], red[3][r][0]));
                const float base = m == -INFINITY ? 0.f : m * a.sl2;
                float ls = 0.f;
                f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (uint32_t v = 0; v < 4; ++v) {
                    const float f = __builtin_amdgcn_exp2f(red[v][r][0] * a.sl2 - base);
                    ls += red[v][r][1] * f;
                    y += *(const f32x4*)(all + (v * 32 + r) * kDim + (g ^ (r & 7)) * 4) * f;
                }
                if (whole) {
                    put_row(a, sp, st.kh, tile0 + r, g, y, m, ls);
                } else {
                    put_part(part + r * kDim + 4 * g, y[0], y[1]);
                    put_part(part + r * kDim + 4 * g + 2, y[2], y[3]);
                    if (g == 0) put_part(part + Sh::kRows * kDim + 2 * r, m, ls);
                }
            }
            if (!whole && last_of_tile()) {
#pragma unroll 1
                for (uint32_t i = tid; i < count * (kDim / 4); i += 256) {
                    const uint32_t r = i / (kDim / 4), g = i % (kDim / 4);
                    if (4 * g >= dim) continue;
                    float m = -INFINITY, ls = 0.f;
                    f32x4 y = {0.f, 0.f, 0.f, 0.f};
                    constexpr uint32_t kAhead = 16;  // parts whose loads are in flight together
#pragma unroll 1
                    for (uint32_t v = w0; v <= w1; v += kAhead) {
                        float2 ml[kAhead], ya[kAhead], yb[kAhead];
#pragma unroll
                        for (uint32_t u = 0; u < kAhead; ++u) {
                            const uint32_t vu = min(v + u, w1);
                            const float* p = a.part + (size_t)(2 * vu + (vu == w0 ? 1 : 0)) * Sh::kPart;
                            ml[u] = get_part(p + Sh::kRows * kDim + 2 * r);
                            ya[u] = get_part(p + r * kDim + 4 * g);
                            yb[u] = get_part(p + r * kDim + 4 * g + 2);
                        }
#pragma unroll
                        for (uint32_t u = 0; u < kAhead; ++u)
                            if (v + u <= w1) {
                                const float top = fmaxf(m, ml[u].x), base = top == -INFINITY ? 0.f : top * a.sl2;
                                const float fa = __builtin_amdgcn_exp2f(m * a.sl2 - base);
                                const float fb = __builtin_amdgcn_exp2f(ml[u].x * a.sl2 - base);
                                m = top;
                                ls = ls * fa + ml[u].y * fb;
                                y = y * fa + f32x4{ya[u].x, ya[u].y, yb[u].x, yb[u].y} * fb;
                            }
                    }
                    put_row(a, sp, st.kh, tile0 + r, g, y, m, ls);
                }
            }
        }
        __syncthreads();  // LDS is free again
        turn ^= 1;

        done += u1 - u0;
        st.unit = 0;
        if (++st.tile == tiles.count) {
            st.tile = 0;
            if (++st.kh == a.kv.heads) {
                st.kh = 0;
                if (done < st.left) {
                    do {
                        ++st.s;
                        sequence();
                    } while (sp.c == 0 && st.s + 1 < a.sq.count);
                }
            }
        }
    }
}

// Collected weights: a workgroup owns kWeightKeys entries of one (sequence, kv
// head), 32 a wave, and adds the probabilities of all rows that see them, in
// order: S = Q K^T (rows down, keys across, so that a lane sums its own key),
// p = exp(scale S - lse).  K is read once and stays in registers; the rows pass
// through LDS 32 at a time, one tile in flight, for the four waves together.
// A launch of its own, since a weight needs its row's whole sum; without atomics.
// Where chains of tiles are long (in_groups) kGroups groups of four waves take the tiles of rows
// in turn, over the same entries, and their sums are added in order: a tile is a chain of load,
// products and weights, and one group's fill another's gaps.
// Measured: single tokens of 8 sequences over 4096 to 12000 entries, 32 + 8 heads of
// 128, 35 us (3.5 TB/s of K); 21 mixed sequences of up to 701 new tokens over up to
// 5003 entries (28 + 4 heads of 80, I8) 261 us of the whole call with one group and
// 143 with four; a chunk of 256 over 6000 in bfloat16 116 and 109.  (A step of 32 rows
// with one group is its chain's latency: deeper rings of loads did not help.)
constexpr uint32_t kWeightKeys = 128;
template <typename T, typename C, uint32_t kDim, uint32_t kGroups>
__global__ __launch_bounds__(256 * kGroups) void weights_tile(TileArgs a, const float* __restrict__ lse, const float* w_in,
                                                    float* w_out, size_t w_seq, size_t w_head) {
    typedef typename Mma<T>::V8 V8;
    constexpr uint32_t G = kDim / 8, kT = kDim / 16, kGranules = 32 * G;  // of 32 keys or rows
    constexpr uint32_t kLoadsK = kGranules / 64, kLoadsQ = kGranules / 256, kStep = 64 / G;
    // K of a group's waves, then two tiles of rows a group (in K's place where there are several: loads
    // to LDS stay below 64 KB)
    constexpr uint32_t kTiles = kGroups > 1 ? 0 : 4;
    __shared__ __attribute__((aligned(65536))) u32x4 lds[(kGroups > 1 ? 2 * kGroups : 6) * kGranules];
    __shared__ __attribute__((aligned(16))) float row_lse[kGroups][2][32];
    __shared__ uint32_t row_lim[kGroups][2][32];
    __shared__ float sums[kGroups > 1 ? kGroups : 1][kWeightKeys];
    const uint32_t tid = threadIdx.x & 255, lane = tid & 63, col = lane & 31, half = lane >> 5;
    const uint32_t group = uniform(threadIdx.x >> 8), wave = uniform(tid >> 6);  // (of the group)
    const uint32_t kh = blockIdx.y, s = blockIdx.z, live = a.kv.dim / 8;
    SeqSpan sp = seq_span(a.sq, a.kv.shift, s, a.tokens);
    sp = {uniform(sp.q0), uniform(sp.c), uniform(sp.n)};
    const uint32_t first = blockIdx.x * kWeightKeys, j0 = first + 32 * wave, j = j0 + col;
    if (first >= sp.n) return;
    const int64_t base = (int64_t)sp.n - sp.c;
    const uint32_t rows = sp.c * a.grp;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
    const u32x4* const zero = &kZeroGranule;
    if (group == 0) {
        typedef typename Held<C>::S S;
        const S* const kb = (const S*)a.kv.K + (size_t)kh * a.kv.kh;
        size_t page[kLoadsK];  // (all looked up before the first load waits for its own)
#pragma unroll
        for (uint32_t i = 0; i < kLoadsK; ++i) page[i] = seq_page(a.sq, a.kv, s, min(j0 + kStep * i + lane / G, sp.n - 1));
#pragma unroll
        for (uint32_t i = 0; i < kLoadsK; ++i) {
            const uint32_t r = kStep * i + lane / G, g = k_at<kDim>(r, lane % G) % G;
            const uint32_t at = min(j0 + r, sp.n - 1) & ((1u << a.kv.shift) - 1);
            const void* const from = g < live ? (const void*)(kb + page[i] * a.kv.kp + at * a.kv.ke + 8 * g) : zero;
            if (Held<C>::k8)
                lds[wave * kGranules + 64 * i + lane] = __builtin_bit_cast(
                    u32x4, widen<C>(*(const u32x2*)from, power(a.kv.kx[page[i] * a.kv.kxp + (size_t)kh * a.kv.kxh + at * a.kv.kxe])));
            else
                load_lds(from, lds0 + 16 * (wave * kGranules + 64 * i));
        }
    }
    // rows of the first token that sees entry `first`, from a whole 32 on
    uint32_t r0 = (first > base ? (uint32_t)((int64_t)first - base) * a.grp / 32 * 32 : 0u) + 32 * group, stage = 0;
    auto load = [&](uint32_t r, uint32_t to) {
#pragma unroll
        for (uint32_t i = 0; i < kLoadsQ; ++i) {
            const uint32_t at = kStep * (kLoadsQ * wave + i) + lane / G, g = k_at<kDim>(at, lane % G) % G, row = r + at;
            const uint32_t tok = row / a.grp, head = kh * a.grp + row % a.grp;
            const T* qr = (const T*)a.q.p + (size_t)(sp.q0 + tok) * a.q.token + (size_t)head * a.q.head;
            load_lds(g < live && row < rows ? (const void*)(qr + 8 * g) : zero,
                     lds0 + 16 * ((kTiles + 2 * group + to) * kGranules + 64 * (kLoadsQ * wave + i)));
        }
    };
    // of row r + tid (32 threads): what is taken from its scores, and the entries that it sees
    float z = INFINITY;
    uint32_t lim = 0;
    auto about = [&](uint32_t r) {
        const uint32_t row = r + tid, tok = row / a.grp, head = kh * a.grp + row % a.grp;
        z = INFINITY;
        lim = 0;
        if (tid < 32 && row < rows) {
            const int64_t see = base + tok + 1;
            lim = see > 0 ? (uint32_t)see : 0u;
            z = lse[(size_t)(sp.q0 + tok) * a.heads + head] * kLog2e;
            if (z == -INFINITY) z = INFINITY;  // a row without a sum gives nothing
        }
    };
    float sum = 0.f, sum2 = 0.f;
    V8 k[kT];
    if (kGroups == 1 && r0 < rows) load(r0, 0);
    wait_loads<0>();
    if (kGroups > 1) __syncthreads();
#pragma unroll
    for (uint32_t t = 0; t < kT; ++t)  // (a negative scale: its sign goes to K here)
        k[t] = __builtin_bit_cast(V8, lds[wave * kGranules + k_at<kDim>(col, 2 * t + half)] ^ a.flip);
    if (kGroups > 1) {
        wait_reads();
        __syncthreads();  // (K's place is free)
        if (r0 - 32 * group < rows) load(r0, 0);
    }
    about(r0);
    // (as many tiles for every group: those beyond the rows are zeros, and seen by nobody)
#pragma unroll 1
    for (; r0 - 32 * group < rows; r0 += 32 * kGroups) {
        if (tid < 32) row_lse[group][stage][tid] = z, row_lim[group][stage][tid] = lim;
        wait_loads<0>();
        __syncthreads();  // these rows are there, and every wave has passed the other tile
        if (r0 - 32 * group + 32 * kGroups < rows) {
            load(r0 + 32 * kGroups, stage ^ 1);
            about(r0 + 32 * kGroups);
        }
        f32x16 x = {};
        V8 q[kT];
#pragma unroll
        for (uint32_t t = 0; t < kT; ++t)
            q[t] = __builtin_bit_cast(V8, lds[(kTiles + 2 * group + stage) * kGranules + k_at<kDim>(col, 2 * t + half)]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t t = 0; t < kT; ++t) x = Mma<T>::mul(q[t], k[t], x);
        const bool masked = j0 + 32 > row_lim[group][stage][0] || r0 + 32 > rows;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const f32x4 zs = *(const f32x4*)&row_lse[group][stage][8 * i + 4 * half];
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u) {
                float p = __builtin_amdgcn_exp2f(x[4 * i + u] * a.sl2 - zs[u]);
                if (masked && j >= row_lim[group][stage][8 * i + 4 * half + u]) p = 0.f;
                (u & 1 ? sum2 : sum) += p;
            }
        }
        stage ^= 1;
    }
    sum = sum_halves(sum + sum2);
    if (kGroups > 1) {
        if (half == 0) sums[kGroups > 1 ? group : 0][32 * wave + col] = sum;
        __syncthreads();
        if (group) return;
        sum = 0.f;
#pragma unroll
        for (uint32_t g = 0; g < kGroups; ++g) sum += sums[kGroups > 1 ? g : 0][32 * wave + col];
    }
    if (half == 0 && j < sp.n) {
        const size_t o = (size_t)s * w_seq + (size_t)kh * w_head + j;
        w_out[o] = ((int64_t)j < base && w_in ? w_in[o] : 0.f) + sum;
    }
}

constexpr uint32_t kGroups = 512;  // two workgroups a compute unit

template <typename T, typename C, uint32_t kDim, bool kSplit>
hipError_t launch_shape(TileArgs a, hipStream_t s) {
    a.whole_page = (1u << a.kv.shift) >= Shape<T, kDim, kSplit>::kKeys && a.kv.dim == kDim &&
                   a.kv.ke < (1u << 20) && a.kv.ve < (1u << 20) && a.kv.kxe < (1u << 20) && a.kv.vxe < (1u << 20);
    a.by_16 = a.kv.kx && a.kv.dim % 16 == 0 && ((uintptr_t)a.kv.K | (uintptr_t)a.kv.V) % 16 == 0 &&
              (a.kv.kp | a.kv.kh | a.kv.ke | a.kv.vp | a.kv.vh | a.kv.ve) % 16 == 0;
    hipLaunchKernelGGL((attend_tile<T, C, kDim, kSplit>), dim3(kGroups), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T, typename C>
hipError_t launch_type(const TileArgs& a, bool split, hipStream_t s) {
    const uint32_t d = a.kv.dim;
    if (split) {
        if (d <= 64) return launch_shape<T, C, 64, true>(a, s);
        if (d <= 128) return launch_shape<T, C, 128, true>(a, s);
        return launch_shape<T, C, 256, true>(a, s);
    }
    if (d <= 64) return launch_shape<T, C, 64, false>(a, s);
    if (d <= 128) return launch_shape<T, C, 128, false>(a, s);
    return launch_shape<T, C, 256, false>(a, s);
}

inline bool in16(const void* p, size_t a, size_t b, size_t c) { return (uintptr_t)p % 16 == 0 && (a | b | c) % 8 == 0; }

}  // namespace

bool attend_tile_fits(const Rows& q, uint32_t tokens, uint32_t heads, const KvView& kv, const SeqView& sq, bool split) {
    if ((q.type != MVK_TYPE_BF16 && q.type != MVK_TYPE_F16) || kv.dim % 8 || kv.dim > 256 || tokens == 0) return false;
    // granules of eight values: 16 bytes, or 8 of a cache held in 8 bits
    const uintptr_t part = ((uintptr_t)kv.K | (uintptr_t)kv.V) % (kv.kx ? 8 : 16);
    if (!in16(q.p, q.token, q.head, 0) || part || (kv.kp | kv.kh | kv.ke | kv.vp | kv.vh | kv.ve) % 8) return false;
    const uint64_t cap = (uint64_t)sq.width << kv.shift;
    if ((cap + kWeightKeys - 1) / kWeightKeys * 256 >= (1ull << 32)) return false;  // threads of the weights' launch
    typedef Shape<__bf16, 128, true> Tokens;  // (rows and units are the same for every type and dim)
    typedef Shape<__bf16, 128, false> Chunks;
    return split ? units_fit<Tokens::kRows, Tokens::kUnit, Tokens::kExtra>(tokens, heads / kv.heads, kv.heads, sq.count, cap)
                 : units_fit<Chunks::kRows, Chunks::kUnit, Chunks::kExtra>(tokens, heads / kv.heads, kv.heads, sq.count, cap);
}

size_t attend_tile_bytes(const KvView& kv, bool split) {
    const uint32_t dim = kv.dim <= 64 ? 64 : kv.dim <= 128 ? 128 : 256, rows = split ? 32 : 128;
    return (size_t)2 * kGroups * (rows * dim + 2 * rows) * sizeof(float);
}

size_t attend_tile_ctrl_bytes() { return (size_t)kGroups * kCounterStride * sizeof(uint32_t); }

bool attend_tile_split(uint32_t max_new, uint32_t heads, const KvView& kv) {
    return (uint64_t)max_new * (heads / kv.heads) <= 32;
}

namespace {

TileArgs tile_args(const Rows& q, uint32_t tokens, uint32_t heads, const KvView& kv, const SeqView& sq, float scale) {
    TileArgs a = {};
    a.q = q, a.kv = kv, a.sq = sq, a.tokens = tokens, a.heads = heads, a.grp = heads / kv.heads;
    // the sign goes to q; a scale of zero as the least number above it, which no score
    // survives, so that masked places stay at -inf
    const float mag = scale < 0 ? -scale : scale;
    a.sl2 = fmaxf(mag * kLog2e, 0x1p-149f);
    a.flip = scale < 0 ? 0x80008000u : 0u;
    return a;
}

}  // namespace

// Are the collected weights taken by several groups of waves a workgroup?  (blocks: of kWeightKeys
// entries that a table's row holds.)  Groups shorten a chain of tiles.  But a workgroup of them fills
// a compute unit where three of one group fit, so sequences of few rows lose, and one that finds no
// entries costs four times as much.
// Up to 128 dims: groups where the longest chain, about 1 us a tile, takes longer than all tiles
// do on 256 compute units, three at a time, and sequences have rows enough, 192 on average.  The
// whole call by one group and by four, us, 128 dims: 21 mixed sequences of up to 701 new tokens
// (28 + 4 heads) 260 and 139, a chunk of 1000 beside 20 of 32 247 and 193, a prompt of 2048 380 and
// 189, four of them 505 and 415; but 48 single tokens 147 and 338, 47 beside a chunk of 256 220 and
// 415, 48 sequences of 32 new 259 and 390 (312 and 786 with a table 32 times as wide), 16 of 256 574
// and 603 (64 dims: 328 and 403).
// Above: one group's 96 KB of LDS leave room for one workgroup, two groups' 64 KB for two.  By one
// and by two, 256 dims: 48 of 32 new 753 and 645, 16 of 256 1695 and 1347; but 48 single tokens 439
// and 477, 47 beside a chunk 615 and 632, and with a table 32 times as wide 48 of 32 840 and 855, 21
// of up to 200 new 262 and 277.
static bool in_groups(uint64_t tokens, uint64_t grp, uint64_t kv_heads, uint64_t count, uint64_t blocks, uint64_t max_new, uint32_t dim) {
    const double rows = (double)(tokens * grp), launch = (double)(count * kv_heads) * (double)blocks;
    if (dim > 128) return rows >= 96. * (double)count && launch <= 14. * rows;
    // (a bound that is all tokens of several sequences says nothing about one: spread evenly)
    const double most = (double)(count > 1 && max_new >= tokens ? tokens / count : max_new < tokens ? max_new : tokens);
    const double tiles = (rows / 32. + (double)count) * (double)kv_heads * (double)blocks;
    return rows >= 192. * (double)count && most * (double)grp / 32. > tiles / 768.;
}

hipError_t launch_weights_tile(const Rows& q, uint32_t tokens, uint32_t heads, const KvView& kv, const SeqView& sq,
                               float scale, const float* lse, const float* w_in, float* w_out, size_t w_seq,
                               size_t w_head, uint32_t max_new, hipStream_t s) {
    const TileArgs a = tile_args(q, tokens, heads, kv, sq, scale);
    const uint64_t cap = (uint64_t)sq.width << kv.shift;
    const dim3 grid((uint32_t)((cap + kWeightKeys - 1) / kWeightKeys), kv.heads, sq.count);
    // (one launch takes fewer than 2^32 threads)
    const bool many = cap < (1u << 28) && in_groups(tokens, heads / kv.heads, kv.heads, sq.count, grid.x, max_new, kv.dim);
    auto go = [&](auto one, auto several, uint32_t groups) {
        hipLaunchKernelGGL(many ? several : one, grid, dim3(many ? 256 * groups : 256), 0, s, a, lse, w_in, w_out, w_seq, w_head);
        return hipGetLastError();
    };
    auto of = [&](auto t, auto c) {
        typedef decltype(t) T;
        typedef decltype(c) C;
        if (kv.dim <= 64) return go(weights_tile<T, C, 64, 1>, weights_tile<T, C, 64, 4>, 4);
        if (kv.dim <= 128) return go(weights_tile<T, C, 128, 1>, weights_tile<T, C, 128, 4>, 4);
        return go(weights_tile<T, C, 256, 1>, weights_tile<T, C, 256, 2>, 2);
    };
    switch (kv.type) {
        case MVK_TYPE_BF16: return of(__bf16(), __bf16());
        case MVK_TYPE_E4M3: return of(__bf16(), E4M3());
        case MVK_TYPE_I8: return of(__bf16(), I8());
        default: return of(_Float16(), _Float16());
    }
}

hipError_t launch_attend_tile(const Rows& q, uint32_t tokens, uint32_t heads, const KvView& kv, const SeqView& sq,
                              float scale, const Rows& out, float inv_scale, float* lse, bool split, void* ws,
                              uint32_t* counters, hipStream_t s) {
    TileArgs a = tile_args(q, tokens, heads, kv, sq, scale);
    a.out = out;
    a.inv_scale = inv_scale, a.lse = lse, a.part = (float*)ws, a.counters = counters;
    const bool half = out.type == MVK_TYPE_BF16 || out.type == MVK_TYPE_F16;
    a.wide_out = (uintptr_t)out.p % (half ? 8 : 16) == 0 && (out.token | out.head) % 4 == 0;
    switch (kv.type) {
        case MVK_TYPE_BF16: return launch_type<__bf16, __bf16>(a, split, s);
        case MVK_TYPE_E4M3: return launch_type<__bf16, E4M3>(a, split, s);
        case MVK_TYPE_I8: return launch_type<__bf16, I8>(a, split, s);
        default: return launch_type<_Float16, _Float16>(a, split, s);
    }
}

}  // namespace mvk
