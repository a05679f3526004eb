// Rotary positions: the table of cosines and sines, and the rotation of new
// tokens' queries and keys with the append of keys and values to the cache.
//
//   (a, b) -> (a cos - b sin, b cos + a sin)  for every pair of the first rot
//   elements of a head, with the angle pos * f_i; the other elements, and v, pass.
//
// One pass over the data: every element is read once, rotated in 32 bits and
// rounded once.  It is bound by memory, or, for a few tokens, by the launch: 8192
// tokens of 64 + 8 heads of 128 in bfloat16 take 63 us (5.4 TB/s; a large copy has
// 5.2), one token of 32 heads 3.6 us.
#include "kv.h"
#include "mvk_internal.h"

namespace mvk {

namespace {

// Frequencies of one table, in radians a position; passed by value.
struct Freqs {
    double f[MVK_MAX_HEAD_DIM / 2];
};

__global__ __launch_bounds__(256) void rotary_table_kernel(Freqs fr, uint32_t half, uint32_t rows, double mag,
                                                           float* __restrict__ out) {
    const size_t count = (size_t)rows * half;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (size_t)gridDim.x * 256) {
        const uint32_t row = (uint32_t)(i / half), c = (uint32_t)(i % half);
        // 64 bits: at position 2^20 a 32-bit product would be 0.06 radians off
        double sn, cs;
        sincos((double)row * fr.f[c], &sn, &cs);
        out[(size_t)row * 2 * half + c] = (float)(cs * mag);
        out[(size_t)row * 2 * half + half + c] = (float)(sn * mag);
    }
}

template <typename S>
struct Src {
    typedef S T;
    static __device__ __forceinline__ float get(S x, float) { return to_float(x); }
};
template <>
struct Src<Field> {
    typedef uint32_t T;
    static __device__ __forceinline__ float get(uint32_t x, float scale) { return field_lift(x) * scale; }
};

struct RotaryArgs {
    Rows q, k, v, qo;
    KvView kv;
    SeqView sq;
    const int32_t* positions;
    const float* table;
    uint32_t T, heads, dim, rot, table_rows;
    float scale;
    bool has_q, has_kv;
};

__device__ __forceinline__ bool entry_of(const RotaryArgs& a, uint32_t t, uint32_t& page, uint32_t& at) {
    return token_entry(a.sq, a.kv, a.T, t, page, at);
}

// Any dim, rot, strides: one thread per pair (rotated or passed) of a head's row.
template <typename S, typename D, bool kHalf>
__global__ __launch_bounds__(256) void rotary_any(RotaryArgs a) {
    typedef typename Src<S>::T ST;
    const uint32_t rows = (a.has_q ? a.heads : 0) + (a.has_kv ? 2 * a.kv.heads : 0);
    const uint32_t pairs = (a.dim + 1) / 2, per = rows * pairs;
    const size_t count = (size_t)a.T * per;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (size_t)gridDim.x * 256) {
        const uint32_t t = (uint32_t)(i / per), in = (uint32_t)(i % per);
        uint32_t row = in / pairs;
        const uint32_t c = in % pairs;
        const ST* x;
        D* dst;
        bool turn = true;
        const uint32_t nq = a.has_q ? a.heads : 0;
        if (row < nq) {
            x = (const ST*)a.q.p + (size_t)t * a.q.token + (size_t)row * a.q.head;
            dst = (D*)a.qo.p + (size_t)t * a.qo.token + (size_t)row * a.qo.head;
        } else {
            row -= nq;
            uint32_t page, at;
            if (!entry_of(a, t, page, at)) continue;
            if (row < a.kv.heads) {
                x = (const ST*)a.k.p + (size_t)t * a.k.token + (size_t)row * a.k.head;
                dst = (D*)a.kv.K + page * a.kv.kp + row * a.kv.kh + at * a.kv.ke;
            } else {
                row -= a.kv.heads;
                x = (const ST*)a.v.p + (size_t)t * a.v.token + (size_t)row * a.v.head;
                dst = (D*)a.kv.V + page * a.kv.vp + row * a.kv.vh + at * a.kv.ve;
                turn = false;
            }
        }
        const uint32_t half = a.rot / 2;
        if (c < half) {
            const uint32_t e0 = kHalf ? c : 2 * c, e1 = kHalf ? c + half : 2 * c + 1;
            const float u = Src<S>::get(x[e0], a.scale), w = Src<S>::get(x[e1], a.scale);
            float cs = 1.f, sn = 0.f;
            if (turn) {
                const int32_t p = a.positions[t];
                const float* tr = a.table + (size_t)(p < 0 ? 0u : min((uint32_t)p, a.table_rows - 1)) * a.rot;
                cs = tr[c];
                sn = tr[half + c];
            }
            dst[e0] = from_float<D>(turn ? u * cs - w * sn : u);
            dst[e1] = from_float<D>(turn ? w * cs + u * sn : w);
        } else {
            for (uint32_t e = 2 * c; e < a.dim && e < 2 * c + 2; ++e) dst[e] = from_float<D>(Src<S>::get(x[e], a.scale));
        }
    }
}

// Eight consecutive values.
template <typename S>
__device__ __forceinline__ void load8(const typename Src<S>::T* p, float scale, float (&x)[8]) {
    typedef typename Src<S>::T ST;
    constexpr int kPer = 16 / sizeof(ST);
#pragma unroll
    for (int i = 0; i < 8 / kPer; ++i) {
        typedef ST V __attribute__((ext_vector_type(kPer)));
        const V v = ((const V*)p)[i];
#pragma unroll
        for (int k = 0; k < kPer; ++k) x[kPer * i + k] = Src<S>::get(v[k], scale);
    }
}
template <typename D>
__device__ __forceinline__ void store8(D* p, const float (&x)[8]) {
    constexpr int kPer = 16 / sizeof(D);
    typedef D V __attribute__((ext_vector_type(kPer)));
#pragma unroll
    for (int i = 0; i < 8 / kPer; ++i) {
        V v;
#pragma unroll
        for (int k = 0; k < kPer; ++k) v[k] = from_float<D>(x[kPer * i + k]);
        ((V*)p)[i] = v;
    }
}

// dim a multiple of 8, rot of 16, rows of 16-byte granules.  A thread takes 16
// elements, whole pairs with their 8 cosines and sines (the granules c and
// c + rot/16 of a head in the half layout, 2c and 2c + 1 in the interleaved
// one, and beyond rot), of kHeads consecutive heads: with 4 heads the table's
// row, read again by every head otherwise, costs a quarter.
template <typename S, typename D, bool kHalf, int kHeads>
__global__ __launch_bounds__(256) void rotary_wide(RotaryArgs a, uint32_t slots, uint32_t blocks, uint32_t count) {
    typedef typename Src<S>::T ST;
    const uint32_t id = blockIdx.x * 256 + threadIdx.x;
    if (id >= count) return;
    const uint32_t c = id % slots, rest = id / slots, t = rest / blocks, row0 = rest % blocks * kHeads;
    const uint32_t nq = a.has_q ? a.heads : 0, nk = a.has_kv ? a.kv.heads : 0, rows = nq + 2 * nk;
    const bool turns = c < a.rot / 16;
    const uint32_t e0 = 8 * (turns && kHalf ? c : 2 * c), e1 = turns && kHalf ? e0 + a.rot / 2 : e0 + 8;
    const bool two = e1 < a.dim;
    float cs[8], sn[8];
    if (turns && row0 < nq + nk) {
        const int32_t p = a.positions[t];
        const float* tr = a.table + (size_t)(p < 0 ? 0u : min((uint32_t)p, a.table_rows - 1)) * a.rot + 8 * c;
        load8<float>(tr, 1.f, cs);
        load8<float>(tr + a.rot / 2, 1.f, sn);
    }
    uint32_t page = 0, at = 0;
    const bool entry = row0 + kHeads > nq && a.has_kv && entry_of(a, t, page, at);
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
        uint32_t row = row0 + u;
        if (row >= rows || (row >= nq && !entry)) break;
        const ST* x;
        D* y;
        bool turn = turns;
        if (row < nq) {
            x = (const ST*)a.q.p + (size_t)t * a.q.token + (size_t)row * a.q.head;
            y = (D*)a.qo.p + (size_t)t * a.qo.token + (size_t)row * a.qo.head;
        } else if ((row -= nq) < nk) {
            x = (const ST*)a.k.p + (size_t)t * a.k.token + (size_t)row * a.k.head;
            y = (D*)a.kv.K + page * a.kv.kp + row * a.kv.kh + at * a.kv.ke;
        } else {
            row -= nk;
            x = (const ST*)a.v.p + (size_t)t * a.v.token + (size_t)row * a.v.head;
            y = (D*)a.kv.V + page * a.kv.vp + row * a.kv.vh + at * a.kv.ve;
            turn = false;
        }
        float p[8], q[8];
        load8<S>(x + e0, a.scale, p);
        if (two) load8<S>(x + e1, a.scale, q);
        if (turn) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                // pair k of the slot: (p[k], q[k]), or two neighbours of the 16 elements
                float& u0 = kHalf ? p[k] : k < 4 ? p[2 * k] : q[2 * k - 8];
                float& u1 = kHalf ? q[k] : k < 4 ? p[2 * k + 1] : q[2 * k - 7];
                const float v0 = u0, v1 = u1;
                u0 = v0 * cs[k] - v1 * sn[k];
                u1 = v1 * cs[k] + v0 * sn[k];
            }
        }
        store8(y + e0, p);
        if (two) store8(y + e1, q);
    }
}

// Rows of 16-byte granules: data and strides.
inline bool granules(const Rows& r, size_t elem) {
    const size_t per = 16 / elem;
    return (uintptr_t)r.p % 16 == 0 && r.token % per == 0 && r.head % per == 0;
}
inline bool granules(const KvView& kv, size_t elem) {
    const size_t per = 16 / elem;
    return (uintptr_t)kv.K % 16 == 0 && (uintptr_t)kv.V % 16 == 0 &&
           (kv.kp | kv.kh | kv.ke | kv.vp | kv.vh | kv.ve) % per == 0;
}

template <typename S, typename D>
hipError_t launch_any(const RotaryArgs& a, bool half, hipStream_t s) {
    const uint32_t rows = (a.has_q ? a.heads : 0) + (a.has_kv ? 2 * a.kv.heads : 0);
    constexpr size_t se = sizeof(typename Src<S>::T), de = sizeof(D);
    const bool aligned = (uintptr_t)a.table % 16 == 0 && (!a.has_q || (granules(a.q, se) && granules(a.qo, de))) &&
                         (!a.has_kv || (granules(a.k, se) && granules(a.v, se) && granules(a.kv, de)));
    const uint32_t slots = (a.dim + 15) / 16;
    // four heads a thread where that leaves a wave for every SIMD
    const bool many = (uint64_t)a.T * slots * rows >= 4u * 64 * 1024;
    const uint32_t blocks = many ? (rows + 3) / 4 : rows;
    const uint64_t threads = (uint64_t)a.T * slots * blocks;
    if (a.dim % 8 == 0 && a.rot % 16 == 0 && aligned && threads < (1ull << 32) - 256) {
        const dim3 grid((uint32_t)((threads + 255) / 256));
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, slots, blocks, (uint32_t)threads);
            return hipGetLastError();
        };
        if (many) return half ? go(rotary_wide<S, D, true, 4>) : go(rotary_wide<S, D, false, 4>);
        return half ? go(rotary_wide<S, D, true, 1>) : go(rotary_wide<S, D, false, 1>);
    }
    const size_t count = (size_t)a.T * rows * ((a.dim + 1) / 2);
    const uint32_t grid = (uint32_t)(count / 256 + 1 < 65536 ? count / 256 + 1 : 65536);
    if (half) hipLaunchKernelGGL((rotary_any<S, D, true>), dim3(grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((rotary_any<S, D, false>), dim3(grid), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename D>
hipError_t launch_to(const RotaryArgs& a, int src, bool half, hipStream_t s) {
    switch (src) {
        case MVK_TYPE_BF16: return launch_any<__bf16, D>(a, half, s);
        case MVK_TYPE_F16: return launch_any<_Float16, D>(a, half, s);
        case MVK_TYPE_F32: return launch_any<float, D>(a, half, s);
        default: return launch_any<Field, D>(a, half, s);
    }
}

}  // namespace

hipError_t launch_rotary_table(const double* freq, uint32_t half, uint32_t rows, double mag, float* out,
                               hipStream_t s) {
    Freqs fr;
    for (uint32_t i = 0; i < MVK_MAX_HEAD_DIM / 2; ++i) fr.f[i] = i < half ? freq[i] : 0.0;
    const size_t blocks = ((size_t)rows * half + 255) / 256;
    hipLaunchKernelGGL(rotary_table_kernel, dim3((uint32_t)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, s, fr,
                       half, rows, mag, out);
    return hipGetLastError();
}

hipError_t launch_rotary(const Rows* q, const Rows* k, const Rows* v, int src, int dst, uint32_t T, uint32_t heads,
                         uint32_t dim, uint32_t rot, bool half, const int32_t* positions, const float* table,
                         uint32_t table_rows, float scale, const Rows* qo, const KvView* kv, const SeqView* sq,
                         hipStream_t s) {
    RotaryArgs a = {};
    a.T = T, a.heads = heads, a.dim = dim, a.rot = rot, a.table_rows = table_rows, a.scale = scale;
    a.positions = positions, a.table = table;
    if (q) a.q = *q, a.qo = *qo, a.has_q = true;
    if (kv) a.k = *k, a.v = *v, a.kv = *kv, a.sq = *sq, a.has_kv = true;
    switch (dst) {
        case MVK_TYPE_BF16: return launch_to<__bf16>(a, src, half, s);
        case MVK_TYPE_F16: return launch_to<_Float16>(a, src, half, s);
        default: return launch_to<float>(a, src, half, s);
    }
}

}  // namespace mvk
