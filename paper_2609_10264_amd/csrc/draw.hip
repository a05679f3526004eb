// Tokens drawn from rows of logits x by temperature, top-k, top-p and min-p from
// given random numbers.
//
//   w_i = exp((x_i - max x) / temperature)
//
// In the order of falling logits (ties: the lowest index first) top-k, top-p and
// min-p each keep a prefix, so what is kept is the shortest one: the logits above a
// threshold and the first few equal to it.  The order needs no sort: the threshold is
// searched digit by digit of an order-preserving key, by counts (top-k) or by sums of
// weights (top-p).  The token is found by a prefix sum in the order of the vocabulary.
//
// Weights are held as whole multiples of 2^-shift, so that every sum is exact, atomics
// included, and no order of additions decides a token at a border.  (That is their sums: a
// weight itself is within 2^-33 of its exponential, see `weight`.)
//
// A workgroup takes a row.  It is read once for the maxima of 4096 groups of its values,
// four a thread.  What is near the top goes to a list in LDS, from the groups whose maximum
// reaches it, and thresholds and the draw are found there: with top-k, the kth largest
// maximum is a bound that k logits at least reach (and not many more); with min-p alone, its
// border; with top-p alone, a histogram of the weights by the first digit of the key, for
// which the row is read again, says where to cut.  Where the list would not hold them, digits
// of the row's keys are searched until it holds those of one bin, and the token is found by
// sums of the row's parts (1 x 131071 in bfloat16: top-k of 50 13 us, every token 76, top-k of
// 20000 154).  A row then is one compute unit's work, 60 instructions a weight: bound by
// their issue, not by memory.  (Bins of values in place of the first digit: a top-p that the
// list holds 25 -> 38 us at 32000, scattered additions to LDS cost more than equal ones.)
#include "mvk_internal.h"
#include "rowio.h"

namespace mvk {

namespace {

// A logit as a number that compares (least: of no weight, as -inf; a not-a-number compares as
// less than any), its key, which orders as the logit does (0 for -inf and not-a-numbers;
// zeros of either sign are one value), and what a key stands for.
template <typename S>
struct Logit {
    typedef S T;
    typedef float N;
    static __device__ __forceinline__ N least() { return -INFINITY; }
    static __device__ __forceinline__ N number(T x) { return to_float(x); }
    static __device__ __forceinline__ N larger(N a, N b) { return fmaxf(a, b); }
    static __device__ __forceinline__ uint32_t key(N x) {
        const float f = x + 0.f;
        const uint32_t b = __float_as_uint(f);
        if (f != f || b == 0xff800000u) return 0u;
        return b & 0x80000000u ? ~b : b | 0x80000000u;
    }
    // The number of a key, the least finite one at least.
    static __device__ __forceinline__ N number_of(uint32_t k) {
        return __uint_as_float(k < 0x00800000u ? 0xff7fffffu : k & 0x80000000u ? k & 0x7fffffffu : ~k);
    }
    static __device__ __forceinline__ float coarse(uint32_t k) { return number_of(k); }
    static __device__ __forceinline__ double value(uint32_t k, float) { return (double)number_of(k); }
    // The key of a number next to v, below it.
    static __device__ __forceinline__ uint32_t key_below(double v, float) {
        const float f = (float)(v - fabs(v) * 0x1p-20 - 0x1p-100);
        return max(key(fmaxf(f, -3.4028234e38f)), 1u);
    }
};
template <>
struct Logit<Field> {
    typedef uint32_t T;
    typedef int32_t N;
    static __device__ __forceinline__ N least() { return (int32_t)0x80000000; }
    static __device__ __forceinline__ N number(T x) { return (int32_t)(x > kP / 2 ? x - kP : x); }
    static __device__ __forceinline__ N larger(N a, N b) { return max(a, b); }
    static __device__ __forceinline__ uint32_t key(N x) { return (uint32_t)x + 0x80000000u; }
    static __device__ __forceinline__ N number_of(uint32_t k) { return (int32_t)(k - 0x80000000u); }
    static __device__ __forceinline__ float coarse(uint32_t k) { return (float)number_of(k); }
    static __device__ __forceinline__ double value(uint32_t k, float scale) { return (double)number_of(k) * (double)scale; }
    static __device__ __forceinline__ uint32_t key_below(double v, float scale) {
        const double f = floor(v / (double)scale) - 1.;
        return f < -2147483647. ? 1u : key((int32_t)f);
    }
};

// A row's settings.
struct Settings {
    double c;       // log2(e) / temperature
    double p;       // 1: off
    double least;   // of min-p; 0: off
    double u;
    uint32_t k;     // 0: off; 1 where only the largest logit counts
};
__device__ __forceinline__ Settings settings_of(const DrawArgs& a, uint32_t r) {
    Settings s;
    const double t = a.how.temperatures ? (double)a.how.temperatures[r] : a.how.temperature;
    const int32_t k = a.how.top_ks ? a.how.top_ks[r] : a.how.top_k;
    const double p = a.how.top_ps ? (double)a.how.top_ps[r] : a.how.top_p;
    const double m = a.how.min_ps ? (double)a.how.min_ps[r] : a.how.min_p;
    const bool greedy = !(t > 0.);
    s.c = greedy ? 0. : 1.4426950408889634074 / t;
    s.k = greedy ? 1u : k < 1 || (uint32_t)k >= a.n ? 0u : (uint32_t)k;
    s.p = !greedy && p < 1. ? fmax(p, 0.) : 1.;
    s.least = !greedy && m > 0. ? fmin(m, 1.) : 0.;
    const float u = a.u[r];
    s.u = u > 0.f && !greedy ? (double)fminf(u, 0x1.fffffep-1f) : 0.;
    return s;
}

// floor(f z) for 0 <= f < 1, and whether something is left.
__device__ __forceinline__ uint64_t part_of(double f, uint64_t z, bool& left) {
    const uint64_t m = (uint64_t)(f * 0x1p64);  // (exact but for bits below 2^-64)
    left = m * z != 0;
    return __umul64hi(m, z);
}

// Weights of a row's keys in units of 2^-shift.  y = (x - top) log2(e) / temperature is
// rounded to 2^-44; its first 10 bits after the point are looked up, the other 34 go
// into a cubic in 32 bits, which below 2^-10 loses 2^-33 of the weight at most (every token of one
// row of 131071: 76 us, 92 by exp2 in 64 bits; 64 rows with top-p of 0.9 206 and 248).
constexpr uint32_t kTable = 1024;
struct Powers {
    double p[kTable];  // 2^(j / kTable)
};
constexpr Powers powers() {
    Powers t = {};
    for (uint32_t j = 0; j < kTable; ++j) {
        // the series of exp(j ln 2 / kTable), from its last term on
        const double x = j * 0.69314718055994530942 / kTable;
        double s = 1.;
        for (int i = 22; i >= 1; --i) s = 1. + x / i * s;
        t.p[j] = s;
    }
    return t;
}
__device__ const Powers kPowers = powers();
struct Weights {
    double top_value, c;
    const double* table;  // 2^(j / kTable)
    uint32_t top, shift;
    float scale;
};
// (of keys above `floor`; the others have none)
template <typename S>
__device__ __forceinline__ uint64_t weight(const Weights& a, uint32_t key, uint32_t floor = 0) {
    if (key == a.top) return 1ull << a.shift;
    const double y = (Logit<S>::value(key, a.scale) - a.top_value) * a.c;
    if (key <= floor || !(y > -47.) || !(y <= 0.)) return 0;  // (-inf below a +inf; 0 inf: none)
    const uint64_t m = __builtin_bit_cast(uint64_t, y + 384.);  // 256 (1 + m 2^-52): steps of 2^-44
    const uint32_t e = ((uint32_t)(m >> 44) & 0xffu) - 128u + a.shift;
    const float g = (float)(uint32_t)(m >> 2) * 0x1.62e43p-43f;  // (the last 34 bits, times ln 2)
    const float p = __builtin_fmaf(g * g, __builtin_fmaf(g, 1.f / 6.f, 0.5f), g);
    const double t = a.table[(uint32_t)(m >> 34) & (kTable - 1)];
    const double w = __builtin_fma(t, (double)p, t);
    const double z = __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, w) + ((uint64_t)e << 52)) + 0x1p52;
    return __builtin_bit_cast(uint64_t, z) & 0xfffffffffffffull;
}

constexpr uint32_t kThreads = 1024, kWaves = kThreads / 64;
constexpr uint32_t kList = 2048;  // logits of the list: two a thread
constexpr uint32_t kBins = 2048;  // of a digit: two a thread
// Largest top-k by way of the maxima: of 4096 groups of values without an order, the
// kth largest maximum is reached by -4096 ln(1 - k / 4096) values, 1712 here.
constexpr uint32_t kMaxima = 1400;

// A value that all lanes have (to the compiler too, which then keeps it apart from the lanes' own).
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) { return (uint64_t)uniform((uint32_t)(x >> 32)) << 32 | uniform((uint32_t)x); }

// Sums of a wave's lanes up to and with each: within rows of 16 lanes, then by each row's last.
template <int kCtrl, int kRows>
__device__ __forceinline__ uint32_t lanes_before(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, kRows, 0xf, false);
}
template <int kCtrl, int kRows>
__device__ __forceinline__ uint64_t lanes_before(uint64_t x) {
    return (uint64_t)lanes_before<kCtrl, kRows>((uint32_t)(x >> 32)) << 32 | lanes_before<kCtrl, kRows>((uint32_t)x);
}
template <typename N>
__device__ __forceinline__ N wave_incl(N x) {
    x += lanes_before<0x111, 0xf>(x);  // row_shr by 1, 2, 4, 8
    x += lanes_before<0x112, 0xf>(x);
    x += lanes_before<0x114, 0xf>(x);
    x += lanes_before<0x118, 0xf>(x);
    x += lanes_before<0x142, 0xa>(x);  // lane 15 of the row before, to rows 1 and 3
    x += lanes_before<0x143, 0xc>(x);  // lane 31, to rows 2 and 3
    return x;
}
__device__ __forceinline__ uint32_t of_lane(uint32_t x, uint32_t lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, (int)lane); }
__device__ __forceinline__ uint64_t of_lane(uint64_t x, uint32_t lane) {
    return (uint64_t)of_lane((uint32_t)(x >> 32), lane) << 32 | of_lane((uint32_t)x, lane);
}

// A row, by steps of kAhead granules a thread: kVec values from at(step, q) on.
template <typename S>
struct RowOf {
    typedef typename Logit<S>::T T;
    static constexpr uint32_t kVec = 16 / sizeof(T), kAhead = 4;
    const T* x;
    uint32_t n;
    __device__ __forceinline__ uint32_t steps() const { return (n + kVec * kThreads * kAhead - 1) / (kVec * kThreads * kAhead); }
    static __device__ __forceinline__ uint32_t at(uint32_t step, uint32_t q) {
        return ((step * kAhead + q) * kThreads + threadIdx.x) * kVec;
    }
    typedef typename Logit<S>::N N;
    typedef T V __attribute__((ext_vector_type(kVec)));
    typedef T Unaligned __attribute__((ext_vector_type(kVec), aligned(sizeof(T))));
    // kVec values from from(i) on, in one load whatever its alignment is: those of a granule
    // at i, or, where the row ends within it, the row's last ones.
    __device__ __forceinline__ uint32_t from(uint32_t i) const { return n >= kVec ? min(i, n - kVec) : 0u; }
    __device__ __forceinline__ V granule(uint32_t i) const {
        if (n >= kVec) return *(const Unaligned*)(x + from(i));
        V v;  // (fewer than eight in all: the last one again)
#pragma unroll
        for (uint32_t e = 0; e < kVec; ++e) v[e] = x[min(e, n - 1)];
        return v;
    }
    __device__ __forceinline__ void load(uint32_t step, V (&v)[kAhead]) const {
#pragma unroll
        for (uint32_t q = 0; q < kAhead; ++q) v[q] = granule(at(step, q));
    }
    // use(key) for every value, end(i) after those from kBlock i on up to the next: four values a thread,
    // 1024 apart.  (One copy of `use`: what is not needed often would else be most of the program.)
    static constexpr uint32_t kBlock = 4 * kThreads;
    template <typename Use, typename End>
    __device__ __forceinline__ void each(Use use, End end) const {
#pragma unroll 1
        for (uint32_t i0 = 0; i0 < n; i0 += kBlock) {
            T v[4];
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u) v[u] = x[min(i0 + u * kThreads + threadIdx.x, n - 1)];
#pragma unroll 1
            for (uint32_t u = 0; u < 4; ++u) {
                const N f = Logit<S>::number(v[0]);
                v[0] = v[1], v[1] = v[2], v[2] = v[3];
                if (i0 + u * kThreads + threadIdx.x < n) use(f == Logit<S>::least() ? 0u : Logit<S>::key(f));
            }
            end(i0 / kBlock);
        }
    }
};

constexpr uint32_t kMembers = 64;  // of one bin of the list
struct Shared {
    double table[kTable];
    uint64_t mass[kBins];
    uint32_t num[kBins];
    uint32_t key[kList], index[kList];
    uint16_t group[4 * kThreads];
    uint64_t wave_mass[kWaves];
    uint32_t wave_num[kWaves], wave_low[kWaves];
    uint64_t found_above, found_mass;
    uint32_t found_bin, found_num, found_before, low, groups, listed, members;
    uint64_t member_mass[kMembers];
    uint32_t member_key[kMembers], rank[64];
    uint64_t before[64], start[64];
};

// Sums over the workgroup up to and with this thread, and the whole.
template <typename N>
struct Sums {
    N incl, all;
};
template <typename N>
__device__ __forceinline__ Sums<N> group_incl(N (&waves)[kWaves], N x) {
    const uint32_t wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const N mine = wave_incl(x);
    __syncthreads();  // (the sums of the call before have been read)
    if (lane == 63) waves[wave] = mine;
    __syncthreads();
    const N w = lane < kWaves ? waves[lane] : N(0), up = wave_incl(w);
    return {mine + of_lane(up - w, wave), of_lane(up, 63)};
}
struct Scan {
    uint32_t num, all_num;
    uint64_t mass, all_mass;
};
__device__ __forceinline__ Scan group_incl(Shared& sh, uint32_t num, uint64_t mass) {
    const Sums<uint32_t> n = group_incl(sh.wave_num, num);
    const Sums<uint64_t> m = group_incl(sh.wave_mass, mass);
    return {n.incl, n.all, m.incl, m.all};
}

// A threshold: kept are the keys above `key` and the first `ties` of those equal to it.
struct Cut {
    uint32_t key, ties;
};
constexpr Cut kAll = {0u, 0u};  // (keys of 0 have no weight)

// One round of a search: of the bins in sh (bin 0: the largest keys) the one where the sum
// of counts, or of weights, from `above` on reaches `need`.
struct Found {
    bool any;
    uint32_t bin, num;     // it, and its keys
    uint32_t before;       // keys of the bins before it (if there is none, of all)
    uint64_t above, mass;  // the sum before it, and the weight of the bins before it (of all)
};
__device__ __forceinline__ Found find_bin(Shared& sh, bool by_mass, uint64_t need, uint64_t above) {
    const uint32_t b = 2 * threadIdx.x;
    __syncthreads();  // (the bins are filled)
    const uint32_t n0 = sh.num[b], n1 = sh.num[b + 1];
    const uint64_t m0 = sh.mass[b], m1 = sh.mass[b + 1];
    const Scan sc = group_incl(sh, n0 + n1, m0 + m1);
    const uint64_t v0 = by_mass ? m0 : n0, v1 = by_mass ? m1 : n1;
    const uint64_t end = above + (by_mass ? sc.mass : sc.num), mid = end - v1, begin = mid - v0;
    if (begin < need && need <= end) {
        const bool second = mid < need;
        sh.found_bin = b + second;
        sh.found_num = second ? n1 : n0;
        sh.found_above = second ? mid : begin;
        sh.found_before = sc.num - n1 - (second ? 0u : n0);
        sh.found_mass = sc.mass - m1 - (second ? 0u : m0);
    }
    __syncthreads();
    const bool any = above + (by_mass ? sc.all_mass : sc.all_num) >= need;
    return Found{any, uniform(sh.found_bin), uniform(sh.found_num), any ? uniform(sh.found_before) : sc.all_num, uniform(sh.found_above),
                 any ? uniform(sh.found_mass) : sc.all_mass};
}

// The bin of a value, the largest in the first.  (Of not-a-numbers, which infinities make: the first.)
__device__ __forceinline__ uint32_t bin_of(float high, float per, float x) {
    const float b = (high - x) * per;
    return b > 0.f ? (uint32_t)fminf(b, (float)(kBins - 1)) : 0u;
}
// find_bin by counts alone.
__device__ __forceinline__ Found find_count(Shared& sh, uint32_t need) {
    const uint32_t b = 2 * threadIdx.x;
    __syncthreads();
    const uint32_t n0 = sh.num[b], n1 = sh.num[b + 1];
    const Sums<uint32_t> s = group_incl<uint32_t>(sh.wave_num, n0 + n1);
    const uint32_t end = s.incl, all = s.all;
    if (end - n0 - n1 < need && need <= end) sh.found_bin = b + (end - n1 < need);
    __syncthreads();
    return Found{all >= need, sh.found_bin};
}

__device__ __forceinline__ void clear_bins(Shared& sh) {
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < kBins; b += kThreads) sh.num[b] = 0, sh.mass[b] = 0;
    __syncthreads();
}

// Digits of the keys of [lo, hi]: bins of 2^width, the largest keys first.
__device__ __forceinline__ uint32_t width_of(uint32_t lo, uint32_t hi) {
    const int have = 32 - __clz((int)((hi - lo) | 1u));
    return have > 11 ? have - 11 : 0;
}
// The range of one bin of [lo, hi].
__device__ __forceinline__ void enter_bin(uint32_t& lo, uint32_t& hi, uint32_t bin, uint32_t width) {
    const uint32_t span = (1u << width) - 1;
    hi -= bin << width;
    lo = hi - lo > span ? hi - span : lo;
}
// Of the keys equal to one, which have weight w each, how many it takes from `above` to `need`.
__device__ __forceinline__ uint32_t ties_of(uint64_t need, uint64_t above, uint64_t w, uint32_t num) {
    const uint64_t rest = need > above ? need - above : 0u, c = w ? (rest + w - 1) / w : 1u;
    return (uint32_t)(c < num ? c : num);
}

template <typename S>
__global__ __launch_bounds__(kThreads) void draw_row(DrawArgs a, uint32_t shift) {
    typedef RowOf<S> Row;
    constexpr uint32_t kVec = Row::kVec, kAhead = Row::kAhead;
    __shared__ Shared sh;
    const uint32_t tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const double power = kPowers.p[tid];
    for (uint32_t r = blockIdx.x; r < a.R; r += gridDim.x) {
        const Row row = {(const typename Row::T*)a.x.p + (size_t)r * a.x.stride, a.n};
        const Settings s = settings_of(a, r);
        const uint32_t steps = row.steps();

        // The largest key, and this thread's own maxima.
        typedef typename Logit<S>::N N;
        uint32_t mine[kAhead], top = 0, low = 0xffffffffu;
        {
            N best[kAhead];
#pragma unroll
            for (uint32_t q = 0; q < kAhead; ++q) best[q] = Logit<S>::least();
            typename Row::V v[kAhead], next[kAhead];
            row.load(0, v);
#pragma unroll 1
            for (uint32_t st = 0; st < steps; ++st) {
                if (st + 1 < steps) row.load(st + 1, next);
#pragma unroll
                for (uint32_t q = 0; q < kAhead; ++q) {
                    // (a group's maximum is one of its own values: a granule at the row's end repeats some
                    // of the one before it, one beyond has none)
                    const uint32_t i = Row::at(st, q), skip = i < a.n ? i - row.from(i) : kVec;
                    if (skip == 0) {
#pragma unroll
                        for (uint32_t e = 0; e < kVec; ++e) best[q] = Logit<S>::larger(best[q], Logit<S>::number(v[q][e]));
                    } else {
#pragma unroll
                        for (uint32_t e = 0; e < kVec; ++e)
                            best[q] = Logit<S>::larger(best[q], e >= skip ? Logit<S>::number(v[q][e]) : Logit<S>::least());
                    }
                    v[q] = next[q];
                }
            }
#pragma unroll
            for (uint32_t q = 0; q < kAhead; ++q) {
                mine[q] = best[q] == Logit<S>::least() ? 0u : Logit<S>::key(best[q]);
                top = max(top, mine[q]);
                if (mine[q]) low = min(low, mine[q]);
            }
        }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) {
            top = max(top, (uint32_t)__shfl_xor((int)top, d));
            low = min(low, (uint32_t)__shfl_xor((int)low, d));
        }
        sh.table[tid] = power;
        __syncthreads();  // (the row before is done with everything shared)
        if (lane == 0) sh.wave_num[wave] = top, sh.wave_low[wave] = low;
        if (tid == 0) sh.low = 0xffffffffu;
        sh.num[tid] = sh.num[tid + kThreads] = 0;
        __syncthreads();
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) top = max(top, sh.wave_num[w]), low = min(low, sh.wave_low[w]);
        top = uniform(top), low = uniform(low);
        if (top == 0u) {  // no logit above -inf
            if (tid == 0) {
                a.tokens[r] = -1;
                if (a.probs) a.probs[r] = 0.f;
            }
            continue;
        }
        const Weights ws = {Logit<S>::value(top, a.scale), s.c, sh.table, top, shift, a.scale};
        const uint64_t least = (uint64_t)ceil(s.least * (double)(1ull << shift));

        // What is kept: of the list of the keys from `from` on, or, without one, by `cut` on the row.
        uint32_t from = 1, listed = 0;
        Cut cut = kAll;
        uint64_t need_p = 0;  // weight that top-p reaches
        auto part_p = [&](uint64_t z) {
            bool left;
            const uint64_t w = part_of(s.p, z, left) + (left ? 1u : 0u);
            return w ? w : 1u;
        };
        // The list: of the keys from `lo` on, of the groups whose maximum reaches it, or (`every`) of those
        // in [lo, hi], of all groups; false if it does not hold them.
        auto collect = [&](uint32_t lo, uint32_t hi, bool every) {
            __syncthreads();
            if (tid == 0) sh.groups = sh.listed = 0;
            __syncthreads();
#pragma unroll
            for (uint32_t q = 0; q < kAhead; ++q)
                if (every || mine[q] >= lo) sh.group[atomicAdd(&sh.groups, 1u)] = (uint16_t)(q * kThreads + tid);
            __syncthreads();
            const uint32_t groups = uniform(sh.groups);
            if (!every && groups > kList) return false;
            const N least_number = Logit<S>::number_of(lo), most_number = Logit<S>::number_of(hi);
            const uint32_t items = groups * steps;  // granules (2^22 at most)
            constexpr uint32_t kFlight = 4;
#pragma unroll 1
            for (uint32_t it = tid; it < items; it += kFlight * kThreads) {
                typename Row::V v[kFlight];
                uint32_t at[kFlight];
#pragma unroll
                for (uint32_t u = 0; u < kFlight; ++u) {
                    const uint32_t i = min(it + u * kThreads, items - 1), g = sh.group[i % groups];
                    at[u] = (i / groups * kAhead * kThreads + g) * kVec;
                    v[u] = row.granule(at[u]);
                }
#pragma unroll 1
                for (uint32_t u = 0; u < kFlight; ++u) {
                    const typename Row::V x = v[0];
                    const uint32_t own = at[0], first = row.from(own);
#pragma unroll
                    for (uint32_t w = 0; w + 1 < kFlight; ++w) v[w] = v[w + 1], at[w] = at[w + 1];
                    uint32_t hits = 0;
#pragma unroll
                    for (uint32_t e = 0; e < kVec; ++e)
                        hits |= Logit<S>::number(x[e]) >= least_number && Logit<S>::number(x[e]) <= most_number && first + e >= own && first + e < a.n ? 1u << e : 0u;
                    if (it + u * kThreads >= items) hits = 0;
                    while (hits) {
                        const uint32_t e = (uint32_t)__ffs((int)hits) - 1;
                        hits &= hits - 1;
                        const uint32_t to = atomicAdd(&sh.listed, 1u);
                        // (again from memory: an index that is not known when this is compiled)
                        if (to < kList) sh.key[to] = Logit<S>::key(Logit<S>::number(row.x[first + e])), sh.index[to] = first + e;
                    }
                }
            }
            __syncthreads();
            listed = uniform(sh.listed);
            return listed <= kList;
        };
        // The least prefix of the row with `need` keys or units of weight (`of_whole`: with top-p's part of
        // the whole): its cut and its weight (`reach`, where top-p asks for it), or false and where the
        // list begins as soon as that can hold it.
        // By digits of the keys, of the row until the list holds those of one bin.
        uint64_t reach = 0;
        auto search_row = [&](bool by_mass, uint64_t need, bool of_whole) {
            uint32_t lo = 1, hi = top, number = 0;  // number: keys above hi
            uint64_t above = 0, above_mass = 0;
            const bool weigh = s.p < 1.;
            bool in_list = false;
#pragma unroll 1
            for (;;) {
                const uint32_t width = width_of(lo, hi);
                clear_bins(sh);
                auto count = [&](uint32_t key) {
                    if (key < lo || key > hi) return;
                    const uint32_t b = (hi - key) >> width;
                    atomicAdd(&sh.num[b], 1u);
                    if (weigh) atomicAdd((unsigned long long*)&sh.mass[b], (unsigned long long)weight<S>(ws, key));
                };
                if (in_list) {
#pragma unroll 1
                    for (uint32_t e = tid; e < listed; e += kThreads) count(sh.key[e]);
                } else {
                    row.each(count, [](uint32_t) {});
                }
                __syncthreads();
                if (of_whole) {
                    need_p = need = part_p(group_incl<uint64_t>(sh.wave_mass, sh.mass[tid] + sh.mass[tid + kThreads]).all);
                    of_whole = false;
                }
                const Found f = find_bin(sh, by_mass, need, above);
                if (f.any) enter_bin(lo, hi, f.bin, width);
                if (number + f.before + (f.any ? f.num : 0u) <= kList) {
                    from = lo;
                    return false;
                }
                above_mass += f.mass;
                if (!f.any) {  // (fewer keys than top-k asks for)
                    cut = kAll;
                    reach = above_mass;
                    return true;
                }
                number += f.before;
                above = f.above;
                if (width == 0) {
                    const uint64_t w = weight<S>(ws, hi);
                    cut = {hi, ties_of(need, above, by_mass ? w : 1u, f.num)};
                    reach = above_mass + cut.ties * w;
                    return true;
                }
                if (!in_list && f.num <= kList) in_list = collect(lo, hi, true);
            }
        };

        bool list_k = false, list_p = false, list_m = false;  // which settings are left to the list
        bool begun = false;                                   // `from` is known
        if (s.k && s.k <= kMaxima) {
            // The kth largest of the maxima, or a little less: bins by value, of which any
            // order would do, and the least maximum in those that hold k.  (The bins are zero.)
            const float high_f = Logit<S>::coarse(top), per = (float)(kBins - 1) / (high_f - Logit<S>::coarse(low));
            uint32_t b[kAhead];
#pragma unroll
            for (uint32_t q = 0; q < kAhead; ++q) {
                b[q] = bin_of(high_f, per, Logit<S>::coarse(mine[q]));
                if (mine[q]) atomicAdd(&sh.num[b[q]], 1u);
            }
            const Found f = find_count(sh, s.k);
            if (f.any) {
                uint32_t bound = 0xffffffffu;
#pragma unroll
                for (uint32_t q = 0; q < kAhead; ++q)
                    if (mine[q] && b[q] <= f.bin) bound = min(bound, mine[q]);
#pragma unroll
                for (int d = 32; d >= 1; d >>= 1) bound = min(bound, (uint32_t)__shfl_xor((int)bound, d));
                if (lane == 0) atomicMin(&sh.low, bound);
                __syncthreads();
                from = uniform(sh.low);
            }
            begun = true;
        } else if (!s.k && !(s.p < 1.) && least) {
            // (weights next to the border are looked at again)
            from = min(top, Logit<S>::key_below(ws.top_value + ((double)log2f((float)s.least) - 0x1p-16) / s.c, a.scale));
            begun = true;
        }
        bool held = begun && collect(from, top, false);
        if (held) list_k = s.k != 0, list_p = s.p < 1., list_m = !s.k && !list_p;
        // Else by the row: top-k, then top-p of what it leaves.
        if (__builtin_expect(!held && (s.k || s.p < 1.), 0)) {
            bool by_mass = !s.k;
#pragma unroll 1
            for (uint32_t round = 0; round < 2; ++round) {  // (one copy of the code)
                if (!search_row(by_mass, by_mass ? need_p : (uint64_t)s.k, !s.k)) {
                    collect(from, top, false);  // (which holds them)
                    list_k = !by_mass, list_p = s.p < 1.;
                    break;
                }
                if (by_mass || !(s.p < 1.)) break;
                need_p = part_p(reach);
                by_mass = true;
            }
        }

        uint64_t z = 0, want = 0;
        auto draw_of = [&](uint64_t total) {
            bool left;
            z = total;
            want = part_of(s.u, z, left);
        };
        auto put = [&](uint32_t index, uint64_t w) {
            a.tokens[r] = (int32_t)index;
            if (a.probs) a.probs[r] = (float)((double)w / (double)z);
        };

        if (__builtin_expect(list_k || list_p || list_m, 1)) {
            if (listed <= 64) {
                // An entry a lane, in every wave: order, thresholds and draw by comparison with four of
                // them a wave.
                if (wave == 0) sh.rank[lane] = 0, sh.before[lane] = sh.start[lane] = 0;
                __syncthreads();
                const uint32_t j0 = 4 * (uint32_t)__builtin_amdgcn_readfirstlane((int)wave);
                const bool in = lane < listed;
                const uint32_t key = in ? sh.key[lane] : 0u, index = in ? sh.index[lane] : 0xffffffffu;
                const uint64_t v = weight<S>(ws, key);
                uint32_t rank = 0;  // entries before this one in the order of the weights, and their weight
                uint64_t before = 0;
#pragma unroll
                for (uint32_t j = j0; j < j0 + 4; ++j) {  // (lanes without an entry have a key of 0)
                    const uint32_t kj = of_lane(key, j);
                    const uint64_t vj = of_lane(v, j);
                    const bool first = kj > key || (kj == key && of_lane(index, j) < index);
                    rank += first ? 1u : 0u;
                    before += first ? vj : 0u;
                }
                atomicAdd(&sh.rank[lane], rank);
                atomicAdd((unsigned long long*)&sh.before[lane], (unsigned long long)before);
                __syncthreads();
                rank = sh.rank[lane], before = sh.before[lane];
                bool on = in && (!list_k || rank < s.k);
                if (list_p) {
                    uint64_t need = need_p;
                    if (list_k) {
                        // the weight that top-k leaves
                        uint64_t all = on ? before + v : 0u;
#pragma unroll
                        for (int d = 32; d >= 1; d >>= 1) {
                            const uint64_t o = (uint64_t)__shfl_xor((long long)all, d);
                            all = o > all ? o : all;
                        }
                        need = part_p(all);
                    }
                    on = on && before < need;
                }
                const uint64_t w = on && v >= least ? v : 0u;
                const uint64_t total = of_lane(wave_incl(w), 63);
                uint64_t start = 0;  // in the order of the vocabulary
#pragma unroll
                for (uint32_t j = j0; j < j0 + 4; ++j) start += of_lane(index, j) < index ? of_lane(w, j) : 0u;
                atomicAdd((unsigned long long*)&sh.start[lane], (unsigned long long)start);
                __syncthreads();
                start = sh.start[lane];
                draw_of(total);
                if (wave == 0 && w && start <= want && want < start + w) put(index, w);
                continue;
            }
            // two entries of the list a thread
            uint32_t k[2], b[2], at[2];
            uint64_t w[2];
            const float high_f = Logit<S>::coarse(top), per = (float)(kBins - 1) / (high_f - Logit<S>::coarse(from));
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i) {
                const uint32_t e = 2 * tid + i;
                k[i] = e < listed ? sh.key[e] : 0u;
                at[i] = e < listed ? sh.index[e] : 0xffffffffu;
                w[i] = weight<S>(ws, k[i]);
                b[i] = bin_of(high_f, per, Logit<S>::coarse(k[i]));
            }
            uint32_t equal = 0;  // keys equal to the cut's
            const bool by_k = list_k;
            list_k &= listed > s.k;
            if (list_k || list_p) {
                clear_bins(sh);
#pragma unroll
                for (uint32_t i = 0; i < 2; ++i)
                    if (k[i]) {
                        atomicAdd(&sh.num[b[i]], 1u);
                        atomicAdd((unsigned long long*)&sh.mass[b[i]], (unsigned long long)w[i]);
                    }
                __syncthreads();
                const uint32_t n0 = sh.num[2 * tid], n1 = sh.num[2 * tid + 1];
                const uint64_t m0 = sh.mass[2 * tid], m1 = sh.mass[2 * tid + 1];
                const Scan sc = group_incl(sh, n0 + n1, m0 + m1);  // of the bins
                // The cut of the least prefix with `need` keys or units of weight; returns the prefix's weight.
                auto search = [&](bool by_mass, uint64_t need) {
                    const uint64_t end = by_mass ? sc.mass : sc.num, v1 = by_mass ? m1 : n1, v0 = by_mass ? m0 : n0;
                    __syncthreads();
                    if (tid == 0) sh.members = 0;
                    if (end - v1 - v0 < need && need <= end) {
                        const bool second = end - v1 < need;
                        sh.found_bin = 2 * tid + second;
                        sh.found_above = second ? end - v1 : end - v1 - v0;
                        sh.found_mass = sc.mass - m1 - (second ? 0 : m0);
                    }
                    __syncthreads();
                    const uint32_t bin = sh.found_bin, num = sh.num[bin];
                    const uint64_t above = sh.found_above, above_m = sh.found_mass;
                    if (num <= kMembers) {
                        // the bin's keys, a lane each (in every wave): their order by comparison
#pragma unroll
                        for (uint32_t i = 0; i < 2; ++i)
                            if (k[i] && b[i] == bin) {
                                const uint32_t at = atomicAdd(&sh.members, 1u);
                                sh.member_key[at] = k[i];
                                sh.member_mass[at] = w[i];
                            }
                        __syncthreads();
                        const bool in = lane < num;
                        const uint32_t key = in ? sh.member_key[lane] : 0u;
                        const uint64_t v = in ? sh.member_mass[lane] : 0u;
                        uint32_t more = 0, same = 0;
                        uint64_t more_m = 0;
                        for (uint32_t j = 0; j < num; ++j) {
                            const uint32_t kj = sh.member_key[j];
                            if (kj > key) ++more, more_m += sh.member_mass[j];
                            same += kj == key ? 1u : 0u;
                        }
                        const uint64_t start = above + (by_mass ? more_m : more), each = by_mass ? v : 1u;
                        const uint64_t hit = __ballot(in && start < need && need <= start + same * each);
                        const int at = hit ? __ffsll((unsigned long long)hit) - 1 : 0;
                        const uint32_t ties = ties_of(need, start, each, same);
                        cut = {(uint32_t)__shfl((int)key, at), (uint32_t)__shfl((int)ties, at)};
                        equal = (uint32_t)__shfl((int)same, at);
                        return (uint64_t)__shfl((long long)(above_m + more_m + ties * v), at);
                    }
                    // many in one bin: bit by bit of the key
                    uint32_t key = 0;
                    uint64_t got = above, got_m = above_m;
                    for (int bit = 31; bit >= 0; --bit) {
                        const uint32_t trial = key | 1u << bit;
                        uint32_t c = 0;
                        uint64_t m = 0;
#pragma unroll
                        for (uint32_t i = 0; i < 2; ++i)
                            if (k[i] >= trial && b[i] == bin && k[i]) ++c, m += w[i];
                        const Scan at = group_incl(sh, c, m);
                        if (above + (by_mass ? at.all_mass : at.all_num) >= need) key = trial;
                    }
                    uint32_t c = 0, eq = 0;
                    uint64_t m = 0;
#pragma unroll
                    for (uint32_t i = 0; i < 2; ++i)
                        if (b[i] == bin && k[i]) {
                            if (k[i] > key) ++c, m += w[i];
                            eq += k[i] == key ? 1u : 0u;
                        }
                    const Scan over = group_incl(sh, c, m);
                    equal = group_incl<uint32_t>(sh.wave_num, eq).all;
                    got += by_mass ? over.all_mass : over.all_num;
                    got_m += over.all_mass;
                    const uint64_t v = weight<S>(ws, key);
                    cut = {key, ties_of(need, got, by_mass ? v : 1u, equal)};
                    return got_m + cut.ties * v;
                };
                uint64_t reach = sc.all_mass;
                if (list_k) reach = search(false, s.k);
                if (list_p) search(true, by_k ? part_p(reach) : need_p);
            }
            bool on[2] = {k[0] > cut.key, k[1] > cut.key};
            if (cut.ties >= equal) {
                on[0] |= k[0] == cut.key, on[1] |= k[1] == cut.key;
            } else {
                // the first of them: the greatest bound of indices that leaves so many
                uint32_t bound = 0;
                for (int bit = 31; bit >= 0; --bit) {
                    const uint32_t trial = bound | 1u << bit;
                    uint32_t c = 0;
#pragma unroll
                    for (uint32_t i = 0; i < 2; ++i) c += k[i] == cut.key && at[i] < trial ? 1u : 0u;
                    if (group_incl<uint32_t>(sh.wave_num, c).all <= cut.ties) bound = trial;
                }
#pragma unroll
                for (uint32_t i = 0; i < 2; ++i) on[i] |= k[i] == cut.key && at[i] < bound;
            }
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i)
                if (!on[i] || w[i] < least) w[i] = 0;
            // The draw, in the order of the vocabulary: bins of indices, then one bin's entries by comparison.
            const uint32_t have = 32 - __clz((int)a.n), narrow = have > 11 ? have - 11 : 0u;
            clear_bins(sh);
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i)
                if (w[i]) {
                    atomicAdd(&sh.num[at[i] >> narrow], 1u);
                    atomicAdd((unsigned long long*)&sh.mass[at[i] >> narrow], (unsigned long long)w[i]);
                }
            __syncthreads();
            const uint64_t m0 = sh.mass[2 * tid], m1 = sh.mass[2 * tid + 1];
            const Sums<uint64_t> sum = group_incl<uint64_t>(sh.wave_mass, m0 + m1);
            draw_of(sum.all);
            if (tid == 0) sh.members = 0;
            if (sum.incl - m0 - m1 <= want && want < sum.incl) {
                const bool second = sum.incl - m1 <= want;
                sh.found_bin = 2 * tid + second;
                sh.found_above = second ? sum.incl - m1 : sum.incl - m1 - m0;
            }
            __syncthreads();
            const uint32_t bin = sh.found_bin;
            if (sh.num[bin] <= kMembers) {
#pragma unroll
                for (uint32_t i = 0; i < 2; ++i)
                    if (w[i] && at[i] >> narrow == bin) {
                        const uint32_t to = atomicAdd(&sh.members, 1u);
                        sh.member_key[to] = at[i];
                        sh.member_mass[to] = w[i];
                    }
                __syncthreads();
                if (wave) continue;
                const uint32_t num = sh.members, index = lane < num ? sh.member_key[lane] : 0u;
                const uint64_t v = lane < num ? sh.member_mass[lane] : 0u;
                uint64_t start = sh.found_above;
                for (uint32_t j = 0; j < num; ++j)
                    if (sh.member_key[j] < index) start += sh.member_mass[j];
                if (v && start <= want && want < start + v) put(index, v);
                continue;
            }
            // many in one bin: the least bound of indices below which the weight is above `want`
            uint32_t bound = 0;  // the greatest below which it is not
            for (int bit = 31; bit >= 0; --bit) {
                const uint32_t trial = bound | 1u << bit;
                const uint64_t m = group_incl<uint64_t>(sh.wave_mass, (at[0] < trial ? w[0] : 0u) + (at[1] < trial ? w[1] : 0u)).all;
                if (m <= want) bound = trial;
            }
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i)
                if (w[i] && at[i] == bound) put(bound, w[i]);
            continue;
        }

        // By the row: the sums of its parts, two blocks each (2048 parts at most), without and with the
        // first ties, then the part that the token is in.
        clear_bins(sh);
        const uint64_t tie_w = cut.key ? weight<S>(ws, cut.key) : 0u, tie = tie_w < least ? 0u : tie_w;
        {
            uint64_t own = 0;
            uint32_t same = 0;
            const uint32_t tie_key = cut.key ? cut.key : 0xffffffffu;
            Weights over = ws;
            if (cut.key == top) over.top = 0xffffffffu;  // (no key: the ties are counted)
            row.each([&](uint32_t key) {
                const uint64_t w = weight<S>(over, key, cut.key);
                own += w < least ? 0u : w;
                same += key == tie_key ? 1u : 0u;
            }, [&](uint32_t block) {
                const uint64_t of_wave = wave_incl(own);
                if (lane == 63) atomicAdd((unsigned long long*)&sh.mass[block / 2], (unsigned long long)of_wave);
                own = 0;
                if (cut.key) {
                    const uint32_t ties = wave_incl(same);
                    if (lane == 63) atomicAdd(&sh.num[block / 2], ties);
                    same = 0;
                }
            });
        }
        __syncthreads();
        const uint32_t n0 = sh.num[2 * tid], n1 = sh.num[2 * tid + 1];
        const uint32_t tied = group_incl<uint32_t>(sh.wave_num, n0 + n1).incl;  // up to and with this thread's parts
        auto kept_of = [&](uint32_t before, uint32_t num) { return (uint64_t)min(num, cut.ties - min(cut.ties, before)) * tie; };
        const uint64_t m0 = sh.mass[2 * tid] + kept_of(tied - n0 - n1, n0), m1 = sh.mass[2 * tid + 1] + kept_of(tied - n1, n1);
        const Sums<uint64_t> sc = group_incl<uint64_t>(sh.wave_mass, m0 + m1);
        draw_of(sc.all);
        if (sc.incl - m0 - m1 <= want && want < sc.incl) {
            const bool second = sc.incl - m1 <= want;
            sh.found_bin = 2 * tid + second;
            sh.found_above = second ? sc.incl - m1 : sc.incl - m1 - m0;
            sh.found_num = second ? tied - n1 : tied - n1 - n0;
        }
        __syncthreads();
        uint32_t seen = sh.found_num;  // ties before
        uint64_t sum = sh.found_above;
#pragma unroll 1
        for (uint32_t i0 = sh.found_bin * 2 * Row::kBlock; i0 < a.n; i0 += kThreads) {
            const uint32_t i = i0 + tid;
            const N f = i < a.n ? Logit<S>::number(row.x[i]) : Logit<S>::least();
            const uint32_t key = f == Logit<S>::least() ? 0u : Logit<S>::key(f), equal = key == cut.key && key ? 1u : 0u;
            const uint64_t w = key >= cut.key ? weight<S>(ws, key) : 0u;
            const Sums<uint32_t> t = group_incl<uint32_t>(sh.wave_num, equal);
            const bool keep = w >= least && (key > cut.key || (equal && seen + t.incl - 1 < cut.ties));
            seen += t.all;
            const Sums<uint64_t> m = group_incl<uint64_t>(sh.wave_mass, keep ? w : 0u);
            const uint64_t end = sum + m.incl;
            sum += m.all;
            if (keep && end - w <= want && want < end) put(i, w);
            if (sum > want) break;  // (for all alike)
        }
    }
}

}  // namespace

hipError_t launch_draw(const DrawArgs& a, hipStream_t s) {
    uint32_t bits = 17;  // sums of n weights stay below 2^62
    while ((1ull << bits) < a.n) ++bits;
    const dim3 grid(a.R < (1u << 20) ? a.R : 1u << 20);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, a, 61 - bits);
        return hipGetLastError();
    };
    switch (a.x.type) {
        case MVK_TYPE_BF16: return go(draw_row<__bf16>);
        case MVK_TYPE_F16: return go(draw_row<_Float16>);
        case MVK_TYPE_F32: return go(draw_row<float>);
        default: return go(draw_row<Field>);
    }
}

}  // namespace mvk
