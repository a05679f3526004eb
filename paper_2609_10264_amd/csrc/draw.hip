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
// Weights are computed in 64 bits and held as whole multiples of 2^-shift, so that
// every sum is exact, atomics included, and no order of additions decides a token
// at a border.
#include "mvk_internal.h"
#include "rowio.h"

namespace mvk {

namespace {

// A logit's key: orders as the logit does; 0 for not-a-numbers and -inf.  (Zeros of
// either sign are one value.)
template <typename S>
struct Logit {
    typedef S T;
    static __device__ __forceinline__ uint32_t key(T x) {
        const float f = to_float(x) + 0.f;
        const uint32_t b = __float_as_uint(f);
        if (f != f || b == 0xff800000u) return 0u;
        return b & 0x80000000u ? ~b : b | 0x80000000u;
    }
    // (x - top) / T for keys, in 64 bits
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
    double inv_t;   // 1 / temperature; 0 where only the largest logit counts
    bool greedy;
    uint32_t k;     // 0: off
    double p;       // 1: off
    double least;   // of min-p
    double u;
};
__device__ __forceinline__ Settings settings_of(const DrawArgs& a, uint32_t r) {
    Settings s;
    const double t = a.how.temperatures ? (double)a.how.temperatures[r] : a.how.temperature;
    const int32_t k = a.how.top_ks ? a.how.top_ks[r] : a.how.top_k;
    const double p = a.how.top_ps ? (double)a.how.top_ps[r] : a.how.top_p;
    const double m = a.how.min_ps ? (double)a.how.min_ps[r] : a.how.min_p;
    s.greedy = !(t > 0.);
    s.inv_t = s.greedy ? 0. : 1. / t;
    s.k = s.greedy || k < 1 || (uint32_t)k >= a.n ? 0u : (uint32_t)k;
    s.p = !s.greedy && p < 1. ? fmax(p, 0.) : 1.;
    s.least = !s.greedy && m > 0. ? fmin(m, 1.) : 0.;
    const float u = a.u[r];
    s.u = u > 0.f ? (double)fminf(u, 0x1.fffffep-1f) : 0.;
    return s;
}

// floor(f z) and whether something is left, for 0 <= f < 1.
__device__ __forceinline__ uint64_t part_of(double f, uint64_t z, bool& left) {
    const uint64_t m = (uint64_t)(f * 0x1p64);  // (exact but for bits below 2^-64)
    left = m * z != 0;
    return __umul64hi(m, z);
}

// Weight of a key in multiples of 2^-shift.
template <typename S>
__device__ __forceinline__ uint64_t weight(uint32_t key, uint32_t top, double top_value, const Settings& s, float scale, double unit) {
    if (key == top) return (uint64_t)unit;
    if (key == 0u && !__is_same(S, Field)) return 0u;
    const double d = (Logit<S>::value(key, scale) - top_value) * s.inv_t;  // (-inf below a +inf; 0 inf: none)
    return s.greedy || !(d <= 0.) ? 0u : (uint64_t)(exp(d) * unit + 0.5);
}

constexpr uint32_t kThreads = 1024, kWaves = kThreads / 64;

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, s));
    return x;
}
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

// A workgroup a row; each step reads the row again.
template <typename S>
__global__ __launch_bounds__(kThreads) void draw_row(DrawArgs a, double unit) {
    typedef Logit<S> L;
    __shared__ uint64_t mass[256], sums[kWaves];
    __shared__ uint32_t num[256], maxima[kWaves], found[4];
    const uint32_t tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, n = a.n;
    for (uint32_t r = blockIdx.x; r < a.R; r += gridDim.x) {
        const typename L::T* x = (const typename L::T*)a.x.p + (size_t)r * a.x.stride;
        const Settings s = settings_of(a, r);
        uint32_t top = 0;
        for (uint32_t i = tid; i < n; i += kThreads) top = max(top, L::key(x[i]));
        top = wave_max(top);
        __syncthreads();
        if (lane == 0) maxima[wave] = top;
        __syncthreads();
        for (uint32_t w = 0; w < kWaves; ++w) top = max(top, maxima[w]);
        if (top == 0u && !__is_same(S, Field)) {  // no logit above -inf
            if (tid == 0) {
                a.tokens[r] = -1;
                if (a.probs) a.probs[r] = 0.f;
            }
            continue;
        }
        const double top_value = L::value(top, a.scale);
        auto w_of = [&](uint32_t key) { return weight<S>(key, top, top_value, s, a.scale, unit); };
        // Kept: keys above thr, and the first `ties` of those equal to it.
        uint32_t thr = 0, ties = 0xffffffffu;
        // The least prefix with `need` entries (by count) or units of weight: its threshold and ties,
        // and the weight of the whole prefix.
        auto search = [&](bool by_weight, uint64_t need, uint32_t& t, uint32_t& c) {
            uint32_t prefix = 0;
            uint64_t above = 0, above_w = 0;  // of the keys above the prefix's range: what is counted, and their weight
            uint32_t last = 0;
            for (int shift = 24; shift >= 0; shift -= 8) {
                __syncthreads();
                if (tid < 256) mass[tid] = 0, num[tid] = 0;
                __syncthreads();
                for (uint32_t i = tid; i < n; i += kThreads) {
                    const uint32_t k = L::key(x[i]);
                    if (shift < 24 && k >> (shift + 8) != prefix) continue;
                    atomicAdd(&num[k >> shift & 255], 1u);
                    atomicAdd((unsigned long long*)&mass[k >> shift & 255], (unsigned long long)w_of(k));
                }
                __syncthreads();
                if (tid == 0) {
                    uint64_t sum = above, sum_w = above_w;
                    int d = 255;
                    for (; d > 0; --d) {
                        const uint64_t v = by_weight ? mass[d] : num[d];
                        if (sum + v >= need) break;
                        sum += v;
                        sum_w += mass[d];
                    }
                    found[0] = (uint32_t)d;
                    found[1] = num[d];
                    sums[0] = sum;
                    sums[1] = sum_w;
                }
                __syncthreads();
                prefix = prefix << 8 | found[0];
                last = found[1];
                above = sums[0];
                above_w = sums[1];
            }
            t = prefix;
            const uint64_t w = w_of(t), rest = need - above;
            const uint64_t want = by_weight ? (w ? (rest + w - 1) / w : 1u) : rest;
            c = (uint32_t)(want < last ? want : last);
            return above_w + (uint64_t)c * w;
        };
        uint64_t total = 0;
        if (s.k) total = search(false, s.k, thr, ties);
        if (s.p < 1.) {
            if (!s.k) {
                // all weights
                uint64_t mine = 0;
                for (uint32_t i = tid; i < n; i += kThreads) mine += w_of(L::key(x[i]));
                mine = wave_incl(mine);
                __syncthreads();
                if (lane == 63) sums[wave] = mine;
                __syncthreads();
                for (uint32_t w = 0; w < kWaves; ++w) total += sums[w];
            }
            bool left;
            uint64_t need = part_of(s.p, total, left);
            need += left ? 1u : 0u;
            search(true, need ? need : 1u, thr, ties);
        }
        const uint64_t least = (uint64_t)ceil(s.least * unit);
        // the kept weights in the order of the vocabulary: their total, then the token
        uint64_t z = 0, want = 0;
        for (int pass = 0; pass < 2; ++pass) {
            uint32_t seen = 0;  // ties before this block of entries
            uint64_t sum = 0;
            bool done = false;
            for (uint32_t i0 = 0; i0 < n && !done; i0 += kThreads) {
                const uint32_t i = i0 + tid, k = i < n ? L::key(x[i]) : 0u;
                const bool tie = i < n && k == thr;
                const uint64_t b = __ballot(tie);
                __syncthreads();
                if (lane == 0) maxima[wave] = (uint32_t)__popcll(b);
                __syncthreads();
                uint32_t rank = seen + (uint32_t)__popcll(b & ((1ull << lane) - 1));
                for (uint32_t w = 0; w < kWaves; ++w) {
                    if (w < wave) rank += maxima[w];
                    seen += maxima[w];
                }
                const bool keep = i < n && (k > thr || (tie && rank < ties));
                uint64_t w = keep ? w_of(k) : 0u;
                if (w < least) w = 0;
                const uint64_t incl = wave_incl(w);
                if (lane == 63) sums[wave] = incl;
                __syncthreads();
                uint64_t at = sum + incl;
                for (uint32_t v = 0; v < kWaves; ++v) {
                    if (v < wave) at += sums[v];
                    sum += sums[v];
                }
                if (pass == 1 && sum > want) {
                    if (w && at > want && at - w <= want) {
                        a.tokens[r] = (int32_t)i;
                        if (a.probs) a.probs[r] = s.greedy ? 1.f : (float)((double)w / (double)z);
                    }
                    done = true;
                }
            }
            if (pass == 0) {
                bool left;
                z = sum;
                want = s.greedy ? 0u : part_of(s.u, z, left);
            }
        }
    }
}

}  // namespace

size_t draw_bytes(const DrawArgs&) { return 0; }

hipError_t launch_draw(const DrawArgs& a, void*, hipStream_t s) {
    int bits = 0;  // sums of n weights stay below 2^62
    while ((1ull << bits) < a.n) ++bits;
    const double unit = (double)(1ull << (61 - (bits < 17 ? 17 : bits)));
    const dim3 grid(a.R < (1u << 20) ? a.R : 1u << 20);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, a, unit);
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
