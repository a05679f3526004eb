// Rotary positions: the table of cosines and sines, and the rotation of new
// tokens' queries and keys with the append of keys and values to the cache.
//
//   (a, b) -> (a cos - b sin, b cos + a sin)  for every pair of the first rot
//   elements of a head, with the angle pos * f_i; the other elements, and v, pass.
//
// One pass over the data: every element is read once, rotated in 32 bits and
// rounded once.  It is bound by memory, or, for a few tokens, by the launch.
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

// Where token t's entry of the cache lies: false if it has none.
__device__ __forceinline__ bool entry_of(const RotaryArgs& a, uint32_t t, uint32_t& page, uint32_t& at) {
    const uint32_t s = seq_of(a.sq, t);
    const SeqSpan sp = seq_span(a.sq, a.kv.shift, s, a.T);
    const int64_t e = (int64_t)sp.n - sp.c + ((int64_t)t - sp.q0);
    if (t < sp.q0 || t >= sp.q0 + sp.c || e < 0) return false;
    const int32_t pg = a.sq.table[(size_t)s * a.sq.ts + (size_t)(e >> a.kv.shift)];
    if (pg < 0 || (uint32_t)pg >= a.kv.pages) return false;
    page = (uint32_t)pg;
    at = (uint32_t)e & ((1u << a.kv.shift) - 1);
    return true;
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
        const Rows* src;
        D* dst;
        bool turn = true;
        const uint32_t nq = a.has_q ? a.heads : 0;
        if (row < nq) {
            src = &a.q;
            dst = (D*)a.qo.p + (size_t)t * a.qo.token + (size_t)row * a.qo.head;
        } else {
            row -= nq;
            uint32_t page, at;
            if (!entry_of(a, t, page, at)) continue;
            if (row < a.kv.heads) {
                src = &a.k;
                dst = (D*)a.kv.K + page * a.kv.kp + row * a.kv.kh + at * a.kv.ke;
            } else {
                row -= a.kv.heads;
                src = &a.v;
                dst = (D*)a.kv.V + page * a.kv.vp + row * a.kv.vh + at * a.kv.ve;
                turn = false;
            }
        }
        const ST* x = (const ST*)src->p + (size_t)t * src->token + (size_t)row * src->head;
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

template <typename S, typename D>
hipError_t launch_any(const RotaryArgs& a, bool half, hipStream_t s) {
    const uint32_t rows = (a.has_q ? a.heads : 0) + (a.has_kv ? 2 * a.kv.heads : 0);
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
