// The end of a block and the beginning of the next:
//   h = residual + scale * gate * after(x),   out = before(h),
//   rms: v (mean v^2 + eps)^-1/2 w + b,   layer: the same of v - mean v.
//
// A workgroup takes a row and keeps it in registers, so that every input is read
// and every output written once; the sums of a norm go across its waves by way of
// LDS.  Bound by memory for many rows, by the chain load, sums, store for few.
// Values and sums are in 32 bits, in 64 with a FIELD output: its whole numbers are
// chosen next to borders and reach 2^30, beyond what 32 bits hold.  A double rounded by
// way of float to a 16-bit type does not occur (64 bits come with FIELD alone, but for
// residual_out, whose h is a float first: an error of 2^-25 of a step more).
#include "mvk_internal.h"
#include "rowio.h"

namespace mvk {

namespace {

template <typename A>
__device__ __forceinline__ A wave_add(A x) {
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) x += __shfl_xor(x, s);
    return x;
}

// The sum over the workgroup, the same in every thread.  `turn`: which half of `part` (no
// half is written again before every thread has read it: a barrier lies between).
template <typename A>
__device__ __forceinline__ A group_sum(A x, A (*part)[16], uint32_t& turn) {
    const uint32_t wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    x = wave_add(x);
    if (waves == 1) return x;
    A* p = part[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) p[wave] = x;
    __syncthreads();
    A sum = 0;
    for (uint32_t w = 0; w < waves; ++w) sum += p[w];
    return sum;
}

// kEach chunks of eight values a thread: chunk tid, tid + threads, ...
template <typename A, int kEach>
__global__ __launch_bounds__(1024) void block_norm(NormArgs a) {
    typedef typename Eight<A>::V V;
    __shared__ A part[2][16];
    uint32_t turn = 0;
    const uint32_t n = a.n, tid = threadIdx.x, threads = blockDim.x;
    const A share = (A)1 / (A)n;
    auto count = [&](int i) {  // values of chunk i
        const uint32_t at = 8 * (tid + i * threads);
        return at < n ? min(8u, n - at) : 0u;
    };
    auto normed = [&](V (&v)[kEach], const NormView& w) {
        if (w.kind == MVK_NORM_LAYER) {
            A sum = 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i)
#pragma unroll
                for (uint32_t k = 0; k < 8; ++k) sum += v[i][k];  // (zeros beyond the row)
            const A mean = group_sum(sum, part, turn) * share;
#pragma unroll
            for (int i = 0; i < kEach; ++i)
#pragma unroll
                for (uint32_t k = 0; k < 8; ++k) v[i][k] = k < count(i) ? v[i][k] - mean : (A)0;
        }
        A sq = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) sq += v[i][k] * v[i][k];
        const A r = (A)1 / sqrt(group_sum(sq, part, turn) * share + (A)w.eps);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t c = count(i), at = 8 * (tid + i * threads);
            if (!c) continue;
            v[i] *= r;
            if (w.weight) v[i] *= load8<A>(w.weight, w.type, w.wide, at, c, 0.f);
            if (w.bias) v[i] += load8<A>(w.bias, w.type, w.wide, at, c, 0.f);
        }
    };
    for (uint32_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        V v[kEach], h[kEach];
        if (a.x.p) {
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                v[i] = load8<A>(a.x.p, a.x.type, a.x.wide, t * a.x.stride + 8 * (tid + i * threads), count(i), a.x_scale);
        }
        if (a.res.p) {
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                h[i] = load8<A>(a.res.p, a.res.type, a.res.wide, t * a.res.stride + 8 * (tid + i * threads), count(i), 0.f);
        }
        if (a.x.p) {
            if (a.after.on) normed(v, a.after);
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const uint32_t at = 8 * (tid + i * threads), c = count(i);
                if (a.gate.p && c) v[i] *= load8<A>(a.gate.p, a.gate.type, a.gate.wide, t * a.gate.stride + at, c, 0.f);
                v[i] *= (A)a.scale;
                if (a.res.p) v[i] += h[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < kEach; ++i) v[i] = h[i];
        }
        if (a.res_out.p) {
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (count(i))
                    store8<A>(a.res_out.p, a.res_out.type, a.res_out.wide, t * a.res_out.stride + 8 * (tid + i * threads),
                              count(i), v[i], (A)1);
        }
        if (!a.out.p) continue;
        if (a.before.on) normed(v, a.before);
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (count(i))
                store8<A>(a.out.p, a.out.type, a.out.wide, t * a.out.stride + 8 * (tid + i * threads), count(i), v[i],
                          (A)1 / (A)a.out_scale);
    }
}

}  // namespace

hipError_t launch_block_norm(const NormArgs& a, hipStream_t s) {
    // four chunks a thread at most
    const uint32_t chunks = (a.n + 7) / 8;
    uint32_t threads = 64;
    while (threads < 1024 && threads < chunks) threads *= 2;
    const uint32_t each = (chunks + threads - 1) / threads;
    const dim3 grid(a.T < (1u << 20) ? a.T : 1u << 20);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, s, a);
        return hipGetLastError();
    };
    if (a.out.p && a.out.type == MVK_TYPE_FIELD)
        return each == 1 ? go(block_norm<double, 1>) : each == 2 ? go(block_norm<double, 2>) : go(block_norm<double, 4>);
    return each == 1 ? go(block_norm<float, 1>) : each == 2 ? go(block_norm<float, 2>) : go(block_norm<float, 4>);
}

}  // namespace mvk
