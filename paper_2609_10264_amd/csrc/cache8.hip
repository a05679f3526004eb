// A cache held in 8 bits: rotary positions with the append to it, and entries of
// any cache read back as rows.
//
//   (a, b) -> (a cos - b sin, b cos + a sin),  e = least with max |x| <= M 2^e,
//   codes = nearest(x / 2^e)
//
// Queries are rotated in 32 bits, as with other caches.  Keys are rotated in 64: a
// code is chosen next to borders, and what is written then is the nearest code of the
// exact value whatever the order of operations.
#include "kv.h"
#include "mvk_internal.h"
#include "quant.h"

namespace mvk {

namespace {

template <typename S>
struct Source {
    typedef S T;
    static __device__ __forceinline__ float f32(T x, float) { return to_float(x); }
    static __device__ __forceinline__ double f64(T x, float) { return to_double(x); }
};
template <>
struct Source<Field> {
    typedef uint32_t T;
    static __device__ __forceinline__ float f32(T x, float scale) { return field_lift(x) * scale; }
    static __device__ __forceinline__ double f64(T x, float scale) { return (double)field_centred(x) * (double)scale; }
};

struct AppendArgs {
    Rows q, k, v, qo;
    KvView kv;
    SeqView sq;
    const int32_t* positions;
    const float* table;
    uint32_t T, heads, dim, rot, table_rows;  // heads: 0 without q
    float scale;
};

__device__ __forceinline__ uint32_t wave_most(uint32_t x) {
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, s));
    return x;
}

// Any dim, rot and strides: a wave per row of a head (q, k or v), pairs lane, lane + 64, ...
constexpr int kPairs = MVK_MAX_HEAD_DIM / 128;
template <typename S, typename C, bool kHalf>
__global__ __launch_bounds__(256) void append_any(AppendArgs a) {
    typedef Source<S> Src;
    const uint32_t lane = threadIdx.x & 63, rows = a.heads + 2 * a.kv.heads, half = a.rot / 2, pairs = (a.dim + 1) / 2;
    const size_t count = (size_t)a.T * rows;
    for (size_t i = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < count; i += (size_t)gridDim.x * 4) {
        const uint32_t t = (uint32_t)(i / rows);
        uint32_t row = (uint32_t)(i % rows), page = 0, at = 0;
        const bool is_q = row < a.heads;
        if (!is_q && !token_entry(a.sq, a.kv, a.T, t, page, at)) continue;
        const int32_t p = a.rot ? a.positions[t] : 0;
        const float* tr = a.table + (size_t)(p < 0 ? 0u : min((uint32_t)p, a.table_rows - 1)) * a.rot;
        auto place = [&](uint32_t c, uint32_t& e0, uint32_t& e1) {  // elements of pair c
            e0 = kHalf && c < half ? c : 2 * c;
            e1 = kHalf && c < half ? c + half : 2 * c + 1;
        };
        if (is_q) {
            const typename Src::T* x = (const typename Src::T*)a.q.p + (size_t)t * a.q.token + (size_t)row * a.q.head;
            __bf16* y = (__bf16*)a.qo.p + (size_t)t * a.qo.token + (size_t)row * a.qo.head;
            for (uint32_t c = lane; c < pairs; c += 64) {
                uint32_t e0, e1;
                place(c, e0, e1);
                const float u = Src::f32(x[e0], a.scale), w = e1 < a.dim ? Src::f32(x[e1], a.scale) : 0.f;
                const float cs = c < half ? tr[c] : 1.f, sn = c < half ? tr[half + c] : 0.f;
                y[e0] = (__bf16)(c < half ? u * cs - w * sn : u);
                if (e1 < a.dim) y[e1] = (__bf16)(c < half ? w * cs + u * sn : w);
            }
            continue;
        }
        row -= a.heads;
        const bool is_k = row < a.kv.heads;
        if (!is_k) row -= a.kv.heads;
        const Rows& r = is_k ? a.k : a.v;
        const typename Src::T* x = (const typename Src::T*)r.p + (size_t)t * r.token + (size_t)row * r.head;
        uint8_t* y = is_k ? (uint8_t*)a.kv.K + page * a.kv.kp + row * a.kv.kh + at * a.kv.ke
                          : (uint8_t*)a.kv.V + page * a.kv.vp + row * a.kv.vh + at * a.kv.ve;
        int8_t* ex = is_k ? a.kv.kx + page * a.kv.kxp + row * a.kv.kxh + at * a.kv.kxe
                          : a.kv.vx + page * a.kv.vxp + row * a.kv.vxh + at * a.kv.vxe;
        double v[kPairs][2];
        uint32_t top = 0;
        bool finite = true;
#pragma unroll
        for (int n = 0; n < kPairs; ++n) {
            const uint32_t c = lane + 64 * n;
            v[n][0] = v[n][1] = 0;
            if (c >= pairs) continue;
            uint32_t e0, e1;
            place(c, e0, e1);
            const double u = Src::f64(x[e0], a.scale), w = e1 < a.dim ? Src::f64(x[e1], a.scale) : 0.;
            const bool turn = is_k && c < half;
            const double cs = turn ? (double)tr[c] : 1., sn = turn ? (double)tr[half + c] : 0.;
            v[n][0] = turn ? u * cs - w * sn : u;
            v[n][1] = turn ? w * cs + u * sn : w;
            top = max(top, max(top_bits(v[n][0]), top_bits(v[n][1])));
            finite &= is_finite(v[n][0]) && is_finite(v[n][1]);
        }
        int e = row_exponent<C>(wave_most(top));
        const bool lost = __is_same(C, I8) && __ballot(!finite) != 0;
        if (lane == 0) *ex = (int8_t)(lost ? MVK_EXP_NAN : e);
#pragma unroll
        for (int n = 0; n < kPairs; ++n) {
            const uint32_t c = lane + 64 * n;
            if (c >= pairs) continue;
            uint32_t e0, e1;
            place(c, e0, e1);
            uint32_t code = lost ? 0u : Held<C>::codes(scaled<C>(v[n][0], e), scaled<C>(v[n][1], e));
            if (!__is_same(C, I8)) {
                if (!is_finite(v[n][0])) code = (code & 0xff00u) | 0x7fu;
                if (!is_finite(v[n][1])) code = (code & 0xffu) | 0x7f00u;
            }
            y[e0] = (uint8_t)code;
            if (e1 < a.dim) y[e1] = (uint8_t)(code >> 8);
        }
    }
}

template <typename S, typename C>
hipError_t launch_append_to(const AppendArgs& a, bool half, hipStream_t s) {
    const size_t count = (size_t)a.T * (a.heads + 2 * a.kv.heads);
    const dim3 grid((uint32_t)((count + 3) / 4 < (1u << 22) ? (count + 3) / 4 : 1u << 22));
    if (half) hipLaunchKernelGGL((append_any<S, C, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((append_any<S, C, false>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

// Any cache, dim and strides: a thread a value.
template <typename C>
__global__ __launch_bounds__(256) void read_any(KvView kv, SeqView sq, uint32_t T, Rows k, Rows v) {
    typedef Held<C> H;
    typedef typename H::S S;
    const size_t per = (size_t)kv.heads * kv.dim, count = (size_t)T * per;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (size_t)gridDim.x * 256) {
        const uint32_t t = (uint32_t)(i / per), h = (uint32_t)(i % per) / kv.dim, d = (uint32_t)(i % per) % kv.dim;
        uint32_t page, at;
        if (!token_entry(sq, kv, T, t, page, at)) continue;
        if (k.p) {
            const float two = H::k8 ? power(kv.kx[page * kv.kxp + h * kv.kxh + at * kv.kxe]) : 1.f;
            store_as(k.p, k.type, (size_t)t * k.token + (size_t)h * k.head + d,
                     H::get(((const S*)kv.K)[page * kv.kp + h * kv.kh + at * kv.ke + d], two), 1.f);
        }
        if (v.p) {
            const float two = H::k8 ? power(kv.vx[page * kv.vxp + h * kv.vxh + at * kv.vxe]) : 1.f;
            store_as(v.p, v.type, (size_t)t * v.token + (size_t)h * v.head + d,
                     H::get(((const S*)kv.V)[page * kv.vp + h * kv.vh + at * kv.ve + d], two), 1.f);
        }
    }
}

}  // namespace

hipError_t launch_append8(const Rows* q, const Rows& k, const Rows& v, uint32_t T, uint32_t heads, uint32_t dim,
                          uint32_t rot, bool half, const int32_t* positions, const float* table, uint32_t table_rows,
                          float scale, const Rows* qo, const KvView& kv, const SeqView& sq, hipStream_t s) {
    AppendArgs a = {};
    a.k = k, a.v = v, a.kv = kv, a.sq = sq;
    a.positions = positions, a.table = table;
    a.T = T, a.heads = q ? heads : 0, a.dim = dim, a.rot = rot, a.table_rows = table_rows, a.scale = scale;
    if (q) a.q = *q, a.qo = *qo;
    const bool e4m3 = kv.type == MVK_TYPE_E4M3;
    switch (k.type) {
        case MVK_TYPE_BF16: return e4m3 ? launch_append_to<__bf16, E4M3>(a, half, s) : launch_append_to<__bf16, I8>(a, half, s);
        case MVK_TYPE_F16: return e4m3 ? launch_append_to<_Float16, E4M3>(a, half, s) : launch_append_to<_Float16, I8>(a, half, s);
        case MVK_TYPE_F32: return e4m3 ? launch_append_to<float, E4M3>(a, half, s) : launch_append_to<float, I8>(a, half, s);
        default: return e4m3 ? launch_append_to<Field, E4M3>(a, half, s) : launch_append_to<Field, I8>(a, half, s);
    }
}

hipError_t launch_cache_read(const KvView& kv, const SeqView& sq, uint32_t T, const Rows& k, const Rows& v,
                             hipStream_t s) {
    const size_t blocks = ((size_t)T * kv.heads * kv.dim + 255) / 256;
    const dim3 grid((uint32_t)(blocks < (1u << 22) ? blocks : 1u << 22));
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, kv, sq, T, k, v);
        return hipGetLastError();
    };
    switch (kv.type) {
        case MVK_TYPE_BF16: return go(read_any<__bf16>);
        case MVK_TYPE_F16: return go(read_any<_Float16>);
        case MVK_TYPE_F32: return go(read_any<float>);
        case MVK_TYPE_E4M3: return go(read_any<E4M3>);
        default: return go(read_any<I8>);
    }
}

}  // namespace mvk
