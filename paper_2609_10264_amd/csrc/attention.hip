// Attention of new tokens over a paged cache, any dim, type and strides.
//
// New token i (of c) of a sequence of n entries sees entries j <= n - c + i:
//   o = sum_j p_j v_j,   p_j = exp(x_j - max) / sum,   x_j = scale q . k_j
// in one pass with the running maximum and sum.  Exponentials are taken to
// base 2: x log2(e) is what is kept, so that each costs one instruction.
#include <algorithm>

#include "kv.h"
#include "mvk_internal.h"
#include "quant.h"

namespace mvk {

namespace {

constexpr uint32_t kMaxDim = MVK_MAX_HEAD_DIM;

// Orders this wave's LDS writes before its later reads (the wave is the only user).
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) x = fmaxf(x, __shfl_xor(x, s));
    return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) x += __shfl_xor(x, s);
    return x;
}

// One wave per (token, head): 64 keys at a time, each lane one product q . k,
// then each lane the values of dims lane, lane + 64, ...  Only entries that the
// row sees are read.
// C: how the cache holds its values; a row of one held in 8 bits has its power of two.
template <typename C>
__global__ __launch_bounds__(256) void attend_any(Rows q, uint32_t tokens, uint32_t heads, KvView kv, SeqView sq,
                                                  float sl2, Rows out, float inv_scale, float* __restrict__ lse) {
    typedef Held<C> H;
    typedef typename H::Q T;
    typedef typename H::S S;
    __shared__ float sq_[4][kMaxDim], sp_[4][64], sv_[H::k8 ? 4 : 1][64];
    __shared__ size_t so_[4][64];
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    // (no barrier below spans waves)
    for (uint32_t row = blockIdx.x * 4 + wave; row < tokens * heads; row += gridDim.x * 4) {
        const uint32_t t = row / heads, h = row % heads, kh = h / (heads / kv.heads), dim = kv.dim;
        const uint32_t s = seq_of(sq, t);
        const SeqSpan sp = seq_span(sq, kv.shift, s, tokens);
        if (t < sp.q0 || t >= sp.q0 + sp.c) continue;
        const int64_t see = (int64_t)sp.n - sp.c + (t - sp.q0) + 1;
        const uint32_t nv = see > 0 ? (uint32_t)see : 0u;
        const T* qr = (const T*)q.p + (size_t)t * q.token + (size_t)h * q.head;
        for (uint32_t d = lane; d < dim; d += 64) sq_[wave][d] = to_float(qr[d]);
        wave_sync();
        float acc[kMaxDim / 64];
#pragma unroll
        for (uint32_t i = 0; i < kMaxDim / 64; ++i) acc[i] = 0.f;
        float m = -INFINITY, l = 0.f;
        for (uint32_t j0 = 0; j0 < nv; j0 += 64) {
            const uint32_t j = j0 + lane, jn = min(64u, nv - j0);
            float x = -INFINITY, two = 1.f;
            size_t off = 0;
            if (j < nv) {
                const size_t page = seq_page(sq, kv, s, j), at = j & ((1u << kv.shift) - 1);
                const S* k = (const S*)kv.K + page * kv.kp + kh * kv.kh + at * kv.ke;
                off = page * kv.vp + kh * kv.vh + at * kv.ve;
                float kt = 1.f;
                if (H::k8) {
                    kt = power(kv.kx[page * kv.kxp + kh * kv.kxh + at * kv.kxe]);
                    two = power(kv.vx[page * kv.vxp + kh * kv.vxh + at * kv.vxe]);
                }
                float d0 = 0.f;
                for (uint32_t d = 0; d < dim; ++d) d0 += sq_[wave][d] * H::get(k[d], kt);
                x = d0 * sl2;
            }
            const float top = wave_max(x), mn = fmaxf(m, top);
            // nothing but -inf so far: keep the sums at zero instead of inf - inf
            const float base = mn == -INFINITY ? 0.f : mn;
            const float p = __builtin_amdgcn_exp2f(x - base), a = __builtin_amdgcn_exp2f(m - base);
            l = l * a + wave_sum(j < nv ? p : 0.f);
            m = mn;
            sp_[wave][lane] = p;
            so_[wave][lane] = off;
            if (H::k8) sv_[H::k8 ? wave : 0][lane] = two;
            wave_sync();
#pragma unroll
            for (uint32_t i = 0; i < kMaxDim / 64; ++i) {
                const uint32_t d = lane + 64 * i;
                if (64 * i < dim) {
                    float o = acc[i] * a;
                    if (d < dim)
                        for (uint32_t u = 0; u < jn; ++u)
                            o += sp_[wave][u] * H::get(((const S*)kv.V)[so_[wave][u] + d], H::k8 ? sv_[H::k8 ? wave : 0][u] : 1.f);
                    acc[i] = o;
                }
            }
            wave_sync();
        }
        const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;  // (a not-a-number stays one)
        if (lse && lane == 0) lse[row] = l > 0.f ? (m + log2f(l)) * kLn2 : l == 0.f ? -INFINITY : l;
#pragma unroll
        for (uint32_t i = 0; i < kMaxDim / 64; ++i) {
            const uint32_t d = lane + 64 * i;
            if (d < dim) store_as(out.p, out.type, (size_t)t * out.token + (size_t)h * out.head + d, acc[i] * inv, inv_scale);
        }
    }
}

// Collected weights: one thread per (sequence, kv head, entry), the rows that
// see the entry in order.
template <typename C>
__global__ __launch_bounds__(256) void weights_any(Rows q, uint32_t tokens, uint32_t heads, KvView kv, SeqView sq,
                                                   float sl2, const float* __restrict__ lse, const float* w_in,
                                                   float* w_out, size_t w_seq, size_t w_head) {
    typedef Held<C> H;
    typedef typename H::Q T;
    typedef typename H::S S;
    const uint32_t kh = blockIdx.y, s = blockIdx.z;
    const SeqSpan sp = seq_span(sq, kv.shift, s, tokens);
    const uint32_t grp = heads / kv.heads;
    for (uint32_t j = blockIdx.x * 256 + threadIdx.x; j < sp.n; j += gridDim.x * 256) {
        const int64_t base = (int64_t)sp.n - sp.c;  // entries before the new tokens
        const size_t page = seq_page(sq, kv, s, j), at = j & ((1u << kv.shift) - 1);
        const S* k = (const S*)kv.K + page * kv.kp + kh * kv.kh + at * kv.ke;
        const float kt = H::k8 ? power(kv.kx[page * kv.kxp + kh * kv.kxh + at * kv.kxe]) : 1.f;
        float sum = 0.f;
        for (uint32_t i = j > base ? (uint32_t)(j - base) : 0u; i < sp.c; ++i)
            for (uint32_t g = 0; g < grp; ++g) {
                const uint32_t t = sp.q0 + i, h = kh * grp + g;
                const T* qr = (const T*)q.p + (size_t)t * q.token + (size_t)h * q.head;
                float d0 = 0.f;
                for (uint32_t d = 0; d < kv.dim; ++d) d0 += to_float(qr[d]) * H::get(k[d], kt);
                const float z = lse[(size_t)t * heads + h];
                sum += z == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(d0 * sl2 - z * kLog2e);
            }
        const size_t o = (size_t)s * w_seq + (size_t)kh * w_head + j;
        w_out[o] = ((int64_t)j < base && w_in ? w_in[o] : 0.f) + sum;
    }
}

}  // namespace

hipError_t launch_attend_any(const Rows& q, uint32_t tokens, uint32_t heads, const KvView& kv, const SeqView& sq,
                             float scale, const Rows& out, float inv_scale, float* lse, hipStream_t s) {
    // (one launch takes fewer than 2^32 threads)
    const dim3 grid((uint32_t)std::min<uint64_t>(((uint64_t)tokens * heads + 3) / 4, 1u << 22));
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, q, tokens, heads, kv, sq, scale * kLog2e, out, inv_scale, lse);
        return hipGetLastError();
    };
    switch (kv.type) {
        case MVK_TYPE_BF16: return go(attend_any<__bf16>);
        case MVK_TYPE_F16: return go(attend_any<_Float16>);
        case MVK_TYPE_E4M3: return go(attend_any<E4M3>);
        case MVK_TYPE_I8: return go(attend_any<I8>);
        default: return go(attend_any<float>);
    }
}

hipError_t launch_weights_any(const Rows& q, uint32_t tokens, uint32_t heads, const KvView& kv, const SeqView& sq,
                              float scale, const float* lse, const float* w_in, float* w_out, size_t w_seq,
                              size_t w_head, hipStream_t s) {
    const uint64_t cap = (uint64_t)sq.width << kv.shift;
    const dim3 grid((uint32_t)((cap + 255) / 256 < 65536 ? (cap + 255) / 256 : 65536), kv.heads, sq.count);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, q, tokens, heads, kv, sq, scale * kLog2e, lse, w_in, w_out,
                           w_seq, w_head);
        return hipGetLastError();
    };
    switch (kv.type) {
        case MVK_TYPE_BF16: return go(weights_any<__bf16>);
        case MVK_TYPE_F16: return go(weights_any<_Float16>);
        case MVK_TYPE_E4M3: return go(weights_any<E4M3>);
        case MVK_TYPE_I8: return go(weights_any<I8>);
        default: return go(weights_any<float>);
    }
}

}  // namespace mvk
