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
// included, and no order of additions decides a token at a border.
//
// A workgroup takes a row.  What is near the top goes, in order, to a list in LDS, on
// which thresholds and the draw are found without the row: with top-k, the kth largest of
// 4096 maxima, four a thread, is a bound that k logits at least reach (and not many more);
// with top-p alone, a histogram of the weights by the first digit of the key says where
// to cut.  The row then is read twice or three times, but once from memory.  Where the
// list would not hold them, the digits of the row's keys are searched to the last.
#include "mvk_internal.h"
#include "rowio.h"

namespace mvk {

namespace {

// A logit's key: orders as the logit does; 0 for not-a-numbers and -inf, which have
// no weight.  (Zeros of either sign are one value.)
template <typename S>
struct Logit {
    typedef S T;
    static __device__ __forceinline__ uint32_t key(T x) {
        const float f = to_float(x) + 0.f;
        const uint32_t b = __float_as_uint(f);
        if (f != f || b == 0xff800000u) return 0u;
        return b & 0x80000000u ? ~b : b | 0x80000000u;
    }
    static __device__ __forceinline__ double value(uint32_t k, float) {
        return (double)__uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
    }
};
template <>
struct Logit<Field> {
    typedef uint32_t T;
    static __device__ __forceinline__ uint32_t key(T x) { return (x > kP / 2 ? x - kP : x) + 0x80000000u; }
    static __device__ __forceinline__ double value(uint32_t k, float scale) {
        return (double)(int32_t)(k - 0x80000000u) * (double)scale;
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
// into a cubic in 32 bits, which below 2^-10 loses 2^-33 of the weight at most.
constexpr uint32_t kTable = 1024;
struct Weights {
    double top_value, c;
    const double* table;  // 2^(j / kTable)
    uint32_t top, shift;
    float scale;
};
template <typename S>
__device__ __forceinline__ uint64_t weight(const Weights& a, uint32_t key) {
    if (key == a.top) return 1ull << a.shift;
    const double y = (Logit<S>::value(key, a.scale) - a.top_value) * a.c;
    if (key == 0u || !(y > -47.) || !(y <= 0.)) return 0;  // (-inf below a +inf; 0 inf: none)
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

template <typename N>
__device__ __forceinline__ N wave_incl(N x) {
    const uint32_t lane = threadIdx.x & 63;
#pragma unroll
    for (uint32_t s = 1; s < 64; s <<= 1) {
        const N y = __shfl_up(x, s);
        if (lane >= s) x += y;
    }
    return x;
}

// A row, by steps of kAhead granules a thread: kVec values from at(step, q) on.
template <typename S>
struct RowOf {
    typedef typename Logit<S>::T T;
    static constexpr uint32_t kVec = 16 / sizeof(T), kAhead = 4;
    const T* x;
    uint32_t n;
    bool wide;
    __device__ __forceinline__ uint32_t steps() const { return (n + kVec * kThreads * kAhead - 1) / (kVec * kThreads * kAhead); }
    static __device__ __forceinline__ uint32_t at(uint32_t step, uint32_t q) {
        return ((step * kAhead + q) * kThreads + threadIdx.x) * kVec;
    }
    // Keys of a step (0 beyond the row), its loads in flight together.
    __device__ __forceinline__ void keys(uint32_t step, uint32_t (&k)[kAhead][kVec]) const {
        typedef T V __attribute__((ext_vector_type(kVec)));
        V v[kAhead];
        if (wide) {
            // (granules that the row does not fill: those of its beginning, or nothing)
            const uint32_t whole = n / kVec * kVec;
#pragma unroll
            for (uint32_t q = 0; q < kAhead; ++q) {
                const uint32_t i = at(step, q);
                if (i < whole) v[q] = *(const V*)(x + i);
                else
#pragma unroll
                    for (uint32_t e = 0; e < kVec; ++e) v[q][e] = x[min(i + e, n - 1)];
            }
        } else {
#pragma unroll
            for (uint32_t q = 0; q < kAhead; ++q)
#pragma unroll
                for (uint32_t e = 0; e < kVec; ++e) v[q][e] = x[min(at(step, q) + e, n - 1)];
        }
#pragma unroll
        for (uint32_t q = 0; q < kAhead; ++q)
#pragma unroll
            for (uint32_t e = 0; e < kVec; ++e) k[q][e] = at(step, q) + e < n ? Logit<S>::key(v[q][e]) : 0u;
    }
};

struct Shared {
    double table[kTable];
    uint64_t mass[kBins];
    uint32_t num[kBins];
    uint32_t key[kList], index[kList];
    uint64_t wave_mass[kWaves];
    uint32_t wave_num[kWaves], counts[2][64];
    uint64_t found_above;
    uint32_t found_bin, found_num, found_key;
};

// Sums over the workgroup up to and with this thread, and the whole.
struct Scan {
    uint32_t num, all_num;
    uint64_t mass, all_mass;
};
__device__ __forceinline__ Scan group_incl(Shared& sh, uint32_t num, uint64_t mass) {
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    Scan r = {wave_incl(num), 0, wave_incl(mass), 0};
    __syncthreads();  // (the sums of the call before have been read)
    if (lane == 63) sh.wave_num[wave] = r.num, sh.wave_mass[wave] = r.mass;
    __syncthreads();
    uint32_t before = 0;
    uint64_t before_m = 0;
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) {
        const uint32_t c = sh.wave_num[w];
        const uint64_t m = sh.wave_mass[w];
        if (w < wave) before += c, before_m += m;
        r.all_num += c, r.all_mass += m;
    }
    r.num += before, r.mass += before_m;
    return r;
}

// A threshold: kept are the keys above `key` and the first `ties` of those equal to it.
struct Cut {
    uint32_t key, ties;
};
constexpr Cut kAll = {0u, 0u};  // (keys of 0 have no weight)

// One digit of a search: of the bins in sh (bin 0: the largest keys) the one where the sum
// of counts, or of weights, from `above` on reaches `need`.
struct Found {
    bool any;
    uint32_t bin, num;  // it, and its keys
    uint64_t above;     // the sum before it
};
__device__ __forceinline__ Found find_bin(Shared& sh, bool by_mass, uint64_t need, uint64_t above) {
    const uint32_t b = 2 * threadIdx.x;
    __syncthreads();  // (the bins are filled)
    const uint32_t n0 = sh.num[b], n1 = sh.num[b + 1];
    const uint64_t v0 = by_mass ? sh.mass[b] : n0, v1 = by_mass ? sh.mass[b + 1] : n1;
    const Scan s = group_incl(sh, 0, v0 + v1);
    const uint64_t end = above + s.mass, mid = end - v1, begin = mid - v0;
    if (begin < need && need <= end) {
        const bool second = mid < need;
        sh.found_bin = b + second;
        sh.found_num = second ? n1 : n0;
        sh.found_above = second ? mid : begin;
    }
    __syncthreads();
    return Found{above + s.all_mass >= need, sh.found_bin, sh.found_num, sh.found_above};
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
    sh.table[tid] = exp2((double)tid / kTable);
    for (uint32_t r = blockIdx.x; r < a.R; r += gridDim.x) {
        const Row row = {(const typename Row::T*)a.x.p + (size_t)r * a.x.stride, a.n, a.x.wide};
        const Settings s = settings_of(a, r);
        const uint32_t steps = row.steps();

        // The largest key, and those of this thread.
        uint32_t mine[kAhead] = {};
#pragma unroll 1
        for (uint32_t st = 0; st < steps; ++st) {
            uint32_t k[kAhead][kVec];
            row.keys(st, k);
#pragma unroll
            for (uint32_t q = 0; q < kAhead; ++q)
#pragma unroll
                for (uint32_t e = 0; e < kVec; ++e) mine[q] = max(mine[q], k[q][e]);
        }
        uint32_t top = max(max(mine[0], mine[1]), max(mine[2], mine[3]));
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
        __syncthreads();  // (the row before is done with everything shared)
        if (lane == 0) sh.wave_num[wave] = top;
        __syncthreads();
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) top = max(top, sh.wave_num[w]);
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
        // The list, in order; false if it does not hold them.
        auto collect = [&]() {
            uint32_t base = 0;
#pragma unroll 1
            for (uint32_t st = 0; st < steps; ++st) {
                uint32_t k[kAhead][kVec], c[kAhead], in[kAhead] = {}, any = 0;
                row.keys(st, k);
#pragma unroll
                for (uint32_t q = 0; q < kAhead; ++q) {
                    c[q] = 0;
#pragma unroll
                    for (uint32_t e = 0; e < kVec; ++e) c[q] += k[q][e] >= from ? 1u : 0u;
                    any |= c[q];
                }
                if (__ballot(any != 0)) {
#pragma unroll
                    for (uint32_t q = 0; q < kAhead; ++q) in[q] = wave_incl(c[q]);
                }
                if (lane == 63) {
#pragma unroll
                    for (uint32_t q = 0; q < kAhead; ++q) sh.counts[st & 1][q * kWaves + wave] = in[q];
                }
                __syncthreads();
                const uint32_t own = sh.counts[st & 1][lane], up = wave_incl(own);
#pragma unroll
                for (uint32_t q = 0; q < kAhead; ++q) {
                    uint32_t to = base + (uint32_t)__shfl((int)(up - own), (int)(q * kWaves + wave)) + in[q] - c[q];
                    if (!c[q]) continue;
#pragma unroll
                    for (uint32_t e = 0; e < kVec; ++e)
                        if (k[q][e] >= from) {
                            if (to < kList) sh.key[to] = k[q][e], sh.index[to] = Row::at(st, q) + e;
                            ++to;
                        }
                }
                base += (uint32_t)__shfl((int)up, 63);
                if (base > kList) break;  // (for all alike)
            }
            __syncthreads();
            listed = base;
            return base <= kList;
        };
        // The least prefix of the row with `need` keys or units of weight (`of_whole`: with top-p's part of
        // the whole): its cut, or false and where the list begins as soon as that can hold it.
        auto search_row = [&](bool by_mass, uint64_t need, bool of_whole) {
            uint32_t lo = 1, hi = top, number = 0;  // number: keys above hi
            uint64_t above = 0;
            for (;;) {
                const uint32_t width = width_of(lo, hi);
                clear_bins(sh);
#pragma unroll 1
                for (uint32_t st = 0; st < steps; ++st) {
                    uint32_t k[kAhead][kVec];
                    row.keys(st, k);
#pragma unroll
                    for (uint32_t q = 0; q < kAhead; ++q)
#pragma unroll
                        for (uint32_t e = 0; e < kVec; ++e) {
                            const uint32_t key = k[q][e];
                            if (key < lo || key > hi) continue;
                            const uint32_t b = (hi - key) >> width;
                            atomicAdd(&sh.num[b], 1u);
                            if (by_mass) atomicAdd((unsigned long long*)&sh.mass[b], (unsigned long long)weight<S>(ws, key));
                        }
                }
                __syncthreads();
                if (of_whole) {
                    need_p = need = part_p(group_incl(sh, 0, sh.mass[tid] + sh.mass[tid + kThreads]).all_mass);
                    of_whole = false;
                }
                const Found f = find_bin(sh, by_mass, need, above);
                const uint32_t past = f.any ? f.bin : kBins - 1;
                uint32_t c = 0;
                for (uint32_t b = tid; b <= past; b += kThreads) c += sh.num[b];
                const uint32_t all = group_incl(sh, c, 0).all_num;
                if (f.any) enter_bin(lo, hi, f.bin, width);
                if (number + all <= kList) {
                    from = lo;
                    return false;
                }
                if (!f.any) {  // (fewer keys than top-k asks for)
                    cut = kAll;
                    return true;
                }
                number += all - f.num;
                above = f.above;
                if (width == 0) {
                    cut = {hi, ties_of(need, above, by_mass ? weight<S>(ws, hi) : 1u, f.num)};
                    return true;
                }
            }
        };

        bool list_k = false, list_p = false;  // which settings are left to the list
        if (s.k) {
            if (s.k <= kMaxima) {
                // the kth largest of the maxima, or a little less
                uint32_t lo = 1, hi = top;
                uint64_t above = 0;
                for (;;) {
                    const uint32_t width = width_of(lo, hi);
                    clear_bins(sh);
#pragma unroll
                    for (uint32_t q = 0; q < kAhead; ++q)
                        if (mine[q] >= lo && mine[q] <= hi) atomicAdd(&sh.num[(hi - mine[q]) >> width], 1u);
                    const Found f = find_bin(sh, false, s.k, above);
                    if (!f.any) break;  // (there are fewer: all of the range)
                    enter_bin(lo, hi, f.bin, width);
                    if (width == 0 || f.above + f.num <= s.k + s.k / 4 + 8) break;
                    above = f.above;
                }
                from = lo;
                list_k = collect();
            }
            if (!list_k) {
                if (!search_row(false, s.k, false)) {
                    list_k = collect();
                } else if (s.p < 1.) {
                    // the weight of what top-k leaves
                    uint64_t z = 0;
#pragma unroll 1
                    for (uint32_t st = 0; st < steps; ++st) {
                        uint32_t k[kAhead][kVec];
                        row.keys(st, k);
#pragma unroll
                        for (uint32_t q = 0; q < kAhead; ++q)
#pragma unroll
                            for (uint32_t e = 0; e < kVec; ++e)
                                if (k[q][e] > cut.key) z += weight<S>(ws, k[q][e]);
                    }
                    need_p = part_p(group_incl(sh, 0, z).all_mass + (uint64_t)cut.ties * weight<S>(ws, cut.key));
                    if (!search_row(true, need_p, false)) list_p = collect();
                }
            }
            list_p |= list_k && s.p < 1.;
        } else if (s.p < 1.) {
            if (!search_row(true, 0, true)) list_p = collect();
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

        if (list_k || list_p) {
            uint32_t k[2];
            uint64_t w[2];
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i) {
                const uint32_t e = tid + i * kThreads;
                k[i] = e < listed ? sh.key[e] : 0u;
                w[i] = weight<S>(ws, k[i]);
            }
            auto search = [&](bool by_mass, uint64_t need) {
                uint32_t lo = from, hi = top;
                uint64_t above = 0;
                for (;;) {
                    const uint32_t width = width_of(lo, hi);
                    clear_bins(sh);
#pragma unroll
                    for (uint32_t i = 0; i < 2; ++i)
                        if (k[i] >= lo && k[i] <= hi) {
                            const uint32_t b = (hi - k[i]) >> width;
                            atomicAdd(&sh.num[b], 1u);
                            if (by_mass) atomicAdd((unsigned long long*)&sh.mass[b], (unsigned long long)w[i]);
                        }
                    const Found f = find_bin(sh, by_mass, need, above);
                    if (!f.any) {
                        cut = kAll;
                        return;
                    }
                    enter_bin(lo, hi, f.bin, width);
                    above = f.above;
                    if (f.num == 1 || width == 0) {
                        // one value: that of whoever has it
#pragma unroll
                        for (uint32_t i = 0; i < 2; ++i)
                            if (k[i] >= lo && k[i] <= hi) sh.found_key = k[i];
                        __syncthreads();
                        const uint32_t key = sh.found_key;
                        cut = {key, ties_of(need, above, by_mass ? weight<S>(ws, key) : 1u, f.num)};
                        return;
                    }
                }
            };
            // (of the list's entries, which are in order) those kept by `cut`
            auto kept = [&](bool (&on)[2]) {
                const Scan first = group_incl(sh, k[0] == cut.key ? 1u : 0u, 0);
                const Scan second = group_incl(sh, k[1] == cut.key ? 1u : 0u, 0);
                on[0] = k[0] > cut.key || (k[0] == cut.key && first.num <= cut.ties);
                on[1] = k[1] > cut.key || (k[1] == cut.key && first.all_num + second.num <= cut.ties);
            };
            bool on[2] = {true, true};  // (places without an entry have no weight)
            if (list_k && listed > s.k) {
                search(false, s.k);
                kept(on);
            }
            if (list_p) {
                if (list_k) need_p = part_p(group_incl(sh, 0, (on[0] ? w[0] : 0) + (on[1] ? w[1] : 0)).all_mass);
                search(true, need_p);
                kept(on);
            }
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i)
                if (!on[i] || w[i] < least) w[i] = 0;
            const Scan first = group_incl(sh, 0, w[0]), second = group_incl(sh, 0, w[1]);
            draw_of(first.all_mass + second.all_mass);
            if (w[0] && first.mass > want && first.mass - w[0] <= want) put(sh.index[tid], w[0]);
            const uint64_t at = first.all_mass + second.mass;
            if (w[1] && at > want && at - w[1] <= want) put(sh.index[tid + kThreads], w[1]);
            continue;
        }

        // On the row: the kept weights in the order of the vocabulary, their total, then the token.
        for (int pass = 0; pass < 2; ++pass) {
            uint32_t seen = 0;  // ties before
            uint64_t sum = 0;
            bool done = false;
#pragma unroll 1
            for (uint32_t st = 0; st < steps && !done; ++st) {
                uint32_t k[kAhead][kVec];
                row.keys(st, k);
#pragma unroll 1
                for (uint32_t q = 0; q < kAhead && !done; ++q) {
                    uint32_t kq[kVec], ties = 0;
#pragma unroll
                    for (uint32_t e = 0; e < kVec; ++e) {
                        kq[e] = k[0][e];
                        ties += kq[e] == cut.key ? 1u : 0u;
                    }
#pragma unroll
                    for (uint32_t v = 0; v + 1 < kAhead; ++v)
#pragma unroll
                        for (uint32_t e = 0; e < kVec; ++e) k[v][e] = k[v + 1][e];
                    const Scan t = group_incl(sh, ties, 0);
                    uint32_t rank = seen + t.num - ties;
                    seen += t.all_num;
                    uint64_t w[kVec], own = 0;
#pragma unroll
                    for (uint32_t e = 0; e < kVec; ++e) {
                        bool keep = kq[e] > cut.key;
                        if (kq[e] == cut.key) keep = rank++ < cut.ties;
                        w[e] = keep ? weight<S>(ws, kq[e]) : 0u;
                        if (w[e] < least) w[e] = 0;
                        own += w[e];
                    }
                    const Scan m = group_incl(sh, 0, own);
                    uint64_t at = sum + m.mass - own;
                    sum += m.all_mass;
                    if (pass == 1 && sum > want) {
#pragma unroll
                        for (uint32_t e = 0; e < kVec; ++e) {
                            if (w[e] && at <= want && at + w[e] > want) put(Row::at(st, q) + e, w[e]);
                            at += w[e];
                        }
                        done = true;
                    }
                }
            }
            if (pass == 0) draw_of(sum);
        }
    }
}

}  // namespace

size_t draw_bytes(const DrawArgs&) { return 0; }

hipError_t launch_draw(const DrawArgs& a, void*, hipStream_t s) {
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
