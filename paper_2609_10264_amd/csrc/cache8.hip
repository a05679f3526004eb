// A cache held in 8 bits: rotary positions with the append to it, and entries of
// any cache read back as rows.
//
//   (a, b) -> (a cos - b sin, b cos + a sin),  e = least with max |x| <= M 2^e,
//   codes = nearest(x / 2^e)
//
// Queries are rotated in 32 bits, as with other caches.  Keys are rotated in 64: a
// code is chosen next to borders, and 64 bits are within 2^-51 of the pair's length of the
// exact value, so that nearly every code is its nearest.
//
// Bound by memory where calls are large: each value is read once and written once.  A
// row's exponent is a maximum over the 4 to 32 neighbouring lanes that hold the row, so
// the append is one pass (8192 tokens of 64 + 8 heads of 128, written and read back: 80 us
// in two launches, 67 and 11, 4.4 TB/s; a wave a row 350).  Rows that are no granules of
// eight values, or whose rotation is none of 16, take a wave a row (2048 tokens of 32 + 8
// heads of 80, half rotated, 50 us with the read; of 128, all rotated, 25).
#include <type_traits>

#include "kv.h"
#include "mvk_internal.h"
#include "quant.h"
#include "rowio.h"

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

// Eight consecutive values.
template <typename S, typename F>
__device__ __forceinline__ void load8_as(const typename Source<S>::T* p, float scale, F (&x)[8]) {
    typedef typename Source<S>::T ST;
    constexpr int kPer = 16 / sizeof(ST);
#pragma unroll
    for (int i = 0; i < 8 / kPer; ++i) {
        typedef ST V __attribute__((ext_vector_type(kPer)));
        const V v = ((const V*)p)[i];
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            if constexpr (__is_same(F, double)) x[kPer * i + k] = Source<S>::f64(v[k], scale);
            else x[kPer * i + k] = Source<S>::f32(v[k], scale);
        }
    }
}

// 16 values of a row, those of `lanes` neighbouring lanes together a whole one, as codes.  (lanes: a
// power of two; values that are not there are zeros.)
template <typename C, typename F>
__device__ __forceinline__ void put_codes(const F (&p)[8], const F (&q)[8], uint32_t lanes, bool first, bool on0, bool on1,
                                          uint8_t* y0, uint8_t* y1, int8_t* ex) {
    uint32_t top = 0;
    bool finite = true;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        top = max(top, max(top_bits(p[k]), top_bits(q[k])));
        finite &= is_finite(p[k]) && is_finite(q[k]);
    }
    uint32_t bad = finite ? 0u : 1u;
    for (uint32_t s = 1; s < lanes; s <<= 1) {
        top = max(top, (uint32_t)__shfl_xor((int)top, (int)s));
        bad |= (uint32_t)__shfl_xor((int)bad, (int)s);
    }
    const int e = row_exponent<C>(top);
    const bool lost = __is_same(C, I8) && bad;
    if (first) *ex = (int8_t)(lost ? MVK_EXP_NAN : e);
    auto codes = [&](const F (&x)[8]) {
        u32x2_ c;
#pragma unroll
        for (int w = 0; w < 2; ++w)
            c[w] = Held<C>::codes(scaled<C>(x[4 * w], e), scaled<C>(x[4 * w + 1], e)) |
                   Held<C>::codes(scaled<C>(x[4 * w + 2], e), scaled<C>(x[4 * w + 3], e)) << 16;
        if (lost) c = u32x2_{0, 0};
        if (!__is_same(C, I8) && bad) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (!is_finite(x[k])) c[k / 4] = (c[k / 4] & ~(0xffu << (8 * (k % 4)))) | 0x7fu << (8 * (k % 4));
        }
        return c;
    };
    if (on0) *(u32x2_*)y0 = codes(p);
    if (on1) *(u32x2_*)y1 = codes(q);
}

// dim a multiple of 8, rot of 16, rows of granules of eight values.  A thread takes 16 elements,
// whole pairs with their cosines and sines (the granules c and c + rot / 16 of a head in the half
// layout, 2c and 2c + 1 in the interleaved one, and beyond rot).  The first `q_blocks` workgroups turn
// queries, kHeads heads a thread; the others write keys and values of one head and token by `lanes`
// neighbouring threads.  Values without a rotation are exact in 32 bits, but for field elements.
template <typename S, typename C, bool kHalf, int kHeads>
__global__ __launch_bounds__(256) void append_wide(AppendArgs a, uint32_t slots, uint32_t q_blocks, uint32_t q_count, uint32_t lanes,
                                                   uint32_t kv_count) {
    typedef typename Source<S>::T ST;
    const bool is_q = blockIdx.x < q_blocks;
    const uint32_t id = (is_q ? blockIdx.x : blockIdx.x - q_blocks) * 256 + threadIdx.x;
    const uint32_t per = is_q ? slots : lanes, c = id % per, rest = id / per;
    const bool turns = c < a.rot / 16;
    const uint32_t e0 = 8 * (turns && kHalf ? c : 2 * c), e1 = turns && kHalf ? e0 + a.rot / 2 : e0 + 8;
    const uint32_t groups = is_q ? (a.heads + kHeads - 1) / kHeads : a.kv.heads;
    const uint32_t t = rest / groups, head0 = rest % groups * (is_q ? kHeads : 1);
    if (id >= (is_q ? q_count : kv_count)) return;  // (whole rows of lanes)
    const bool on0 = e0 < a.dim, on1 = e1 < a.dim;
    typedef float V4 __attribute__((ext_vector_type(4)));
    V4 cs[2] = {}, sn[2] = {};
    if (turns) {
        const int32_t p = a.positions[t];
        const float* tr = a.table + (size_t)(p < 0 ? 0u : min((uint32_t)p, a.table_rows - 1)) * a.rot + 8 * c;
        cs[0] = ((const V4*)tr)[0], cs[1] = ((const V4*)tr)[1];
        sn[0] = ((const V4*)(tr + a.rot / 2))[0], sn[1] = ((const V4*)(tr + a.rot / 2))[1];
    }
    auto turn = [&](auto& p, auto& q) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            // pair k of the slot: (p[k], q[k]), or two neighbours of the 16 elements
            auto& u0 = kHalf ? p[k] : k < 4 ? p[2 * k] : q[2 * k - 8];
            auto& u1 = kHalf ? q[k] : k < 4 ? p[2 * k + 1] : q[2 * k - 7];
            const auto v0 = u0, v1 = u1;
            u0 = v0 * cs[k / 4][k % 4] - v1 * sn[k / 4][k % 4];
            u1 = v1 * cs[k / 4][k % 4] + v0 * sn[k / 4][k % 4];
        }
    };
    if (is_q) {
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
            const uint32_t head = head0 + h;
            if (head >= a.heads || !on0) break;
            const ST* x = (const ST*)a.q.p + (size_t)t * a.q.token + (size_t)head * a.q.head;
            __bf16* y = (__bf16*)a.qo.p + (size_t)t * a.qo.token + (size_t)head * a.qo.head;
            float p[8], q[8];
            load8_as<S>(x + e0, a.scale, p);
            if (on1) load8_as<S>(x + e1, a.scale, q);
            if (turns) turn(p, q);
            typedef __bf16 B8 __attribute__((ext_vector_type(8)));
            B8 b, d;
#pragma unroll
            for (int k = 0; k < 8; ++k) b[k] = (__bf16)p[k], d[k] = (__bf16)q[k];
            *(B8*)(y + e0) = b;
            if (on1) *(B8*)(y + e1) = d;
        }
        return;
    }
    uint32_t page = 0, at = 0;
    if (!token_entry(a.sq, a.kv, a.T, t, page, at)) return;  // (the same for a row's threads)
    const ST* k = (const ST*)a.k.p + (size_t)t * a.k.token + (size_t)head0 * a.k.head;
    const ST* v = (const ST*)a.v.p + (size_t)t * a.v.token + (size_t)head0 * a.v.head;
    uint8_t* ky = (uint8_t*)a.kv.K + page * a.kv.kp + head0 * a.kv.kh + at * a.kv.ke;
    uint8_t* vy = (uint8_t*)a.kv.V + page * a.kv.vp + head0 * a.kv.vh + at * a.kv.ve;
    int8_t* kx = a.kv.kx + page * a.kv.kxp + head0 * a.kv.kxh + at * a.kv.kxe;
    int8_t* vx = a.kv.vx + page * a.kv.vxp + head0 * a.kv.vxh + at * a.kv.vxe;
    {
        double p[8] = {}, q[8] = {};
        if (on0) load8_as<S>(k + e0, a.scale, p);
        if (on1) load8_as<S>(k + e1, a.scale, q);
        if (turns) turn(p, q);
        put_codes<C>(p, q, lanes, c == 0, on0, on1, ky + e0, ky + e1, kx);
    }
    typedef typename std::conditional<std::is_same<S, Field>::value, double, float>::type F;
    F p[8] = {}, q[8] = {};
    if (on0) load8_as<S>(v + e0, a.scale, p);
    if (on1) load8_as<S>(v + e1, a.scale, q);
    put_codes<C>(p, q, lanes, c == 0, on0, on1, vy + e0, vy + e1, vx);
}

// Rows of granules of eight values, which 8 or 16 bytes hold (or two loads of 16).
inline bool kv_granules(const KvView& kv) {
    return ((uintptr_t)kv.K | (uintptr_t)kv.V) % (kv.kx ? 8 : 16) == 0 && (kv.kp | kv.kh | kv.ke | kv.vp | kv.vh | kv.ve) % 8 == 0;
}

template <typename S, typename C>
hipError_t launch_append_to(const AppendArgs& a, bool half, hipStream_t s) {
    constexpr size_t per = 16 / sizeof(typename Source<S>::T);  // values of a load
    auto wide = [&](const Rows& r, size_t each) { return (uintptr_t)r.p % 16 == 0 && (r.token | r.head) % each == 0; };
    const uint32_t slots = (a.dim + 15) / 16;
    uint32_t lanes = 1;
    while (lanes < slots) lanes *= 2;
    const bool many = (uint64_t)a.T * slots * a.heads >= 4u * 64 * 1024;  // (as with other caches)
    const uint64_t q_count = (uint64_t)a.T * slots * (many ? (a.heads + 3) / 4 : a.heads);
    const uint64_t kv_count = (uint64_t)a.T * a.kv.heads * lanes, q_blocks = (q_count + 255) / 256;
    if (a.dim % 8 == 0 && a.rot % 16 == 0 && (uintptr_t)a.table % 16 == 0 && wide(a.k, per) && wide(a.v, per) &&
        (!a.heads || (wide(a.q, per) && wide(a.qo, 8))) && kv_granules(a.kv) && q_count + kv_count < (1ull << 32) - 1024) {
        const dim3 grid((uint32_t)(q_blocks + (kv_count + 255) / 256));
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, slots, (uint32_t)q_blocks, (uint32_t)q_count, lanes,
                               (uint32_t)kv_count);
            return hipGetLastError();
        };
        if (many) return half ? go(append_wide<S, C, true, 4>) : go(append_wide<S, C, false, 4>);
        return half ? go(append_wide<S, C, true, 1>) : go(append_wide<S, C, false, 1>);
    }
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

// Rows of granules of eight values: a thread one of K and of V.
template <typename C>
__global__ __launch_bounds__(256) void read_wide(KvView kv, SeqView sq, uint32_t T, Rows k, Rows v, uint32_t count) {
    typedef Held<C> H;
    const uint32_t id = blockIdx.x * 256 + threadIdx.x, per = kv.dim / 8;
    if (id >= count) return;
    const uint32_t g = id % per, h = id / per % kv.heads, t = id / per / kv.heads;
    uint32_t page, at;
    if (!token_entry(sq, kv, T, t, page, at)) return;
    auto copy = [&](const Rows& to, const void* pool, size_t from, const int8_t* ex, size_t ex_at) {
        if (!to.p) return;
        const size_t i = (size_t)t * to.token + (size_t)h * to.head + 8 * g;
        if constexpr (H::k8) {
            const u32x4q b = widen<C>(*(const u32x2_*)((const uint8_t*)pool + from + 8 * g), power(ex[ex_at]));
            if (to.type == MVK_TYPE_BF16) {
                *(u32x4q*)((uint16_t*)to.p + i) = b;
            } else {
                Raw8 r;
                r.lo = r.hi = b;
                store8<float>(to.p, to.type, i, values_of<float>(r, MVK_TYPE_BF16, 0.f), 1.f);
            }
        } else {
            constexpr int type = __is_same(C, __bf16) ? MVK_TYPE_BF16 : __is_same(C, _Float16) ? MVK_TYPE_F16 : MVK_TYPE_F32;
            store8<float>(to.p, to.type, i, values_of<float>(load_raw8(pool, type, from + 8 * g), type, 0.f), 1.f);
        }
    };
    copy(k, kv.K, page * kv.kp + h * kv.kh + at * kv.ke, kv.kx, page * kv.kxp + h * kv.kxh + at * kv.kxe);
    copy(v, kv.V, page * kv.vp + h * kv.vh + at * kv.ve, kv.vx, page * kv.vxp + h * kv.vxh + at * kv.vxe);
}

template <typename C>
hipError_t launch_read_of(const KvView& kv, const SeqView& sq, uint32_t T, const Rows& k, const Rows& v, hipStream_t s) {
    auto wide = [](const Rows& r) {
        const size_t per = r.type == MVK_TYPE_F32 ? 4 : 8;
        return !r.p || ((uintptr_t)r.p % 16 == 0 && (r.token | r.head) % per == 0);
    };
    const uint64_t count = (uint64_t)T * kv.heads * (kv.dim / 8);
    if (kv.dim % 8 == 0 && kv_granules(kv) && wide(k) && wide(v) && count < (1ull << 32) - 256) {
        hipLaunchKernelGGL(read_wide<C>, dim3((uint32_t)((count + 255) / 256)), dim3(256), 0, s, kv, sq, T, k, v, (uint32_t)count);
        return hipGetLastError();
    }
    const size_t blocks = ((size_t)T * kv.heads * kv.dim + 255) / 256;
    hipLaunchKernelGGL(read_any<C>, dim3((uint32_t)(blocks < (1u << 22) ? blocks : 1u << 22)), dim3(256), 0, s, kv, sq, T, k, v);
    return hipGetLastError();
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
    switch (kv.type) {
        case MVK_TYPE_BF16: return launch_read_of<__bf16>(kv, sq, T, k, v, s);
        case MVK_TYPE_F16: return launch_read_of<_Float16>(kv, sq, T, k, v, s);
        case MVK_TYPE_F32: return launch_read_of<float>(kv, sq, T, k, v, s);
        case MVK_TYPE_E4M3: return launch_read_of<E4M3>(kv, sq, T, k, v, s);
        default: return launch_read_of<I8>(kv, sq, T, k, v, s);
    }
}

}  // namespace mvk
