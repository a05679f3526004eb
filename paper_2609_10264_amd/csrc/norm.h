// The end of a block and the beginning of the next:
//   h = residual + scale * gate * after(x),   out = before(h),
//   rms: v (mean v^2 + eps)^-1/2 w + b,   layer: the same of v - mean v.
//
// A workgroup takes a row and keeps it in registers, so that every input is read
// and every output written once; the sums of a norm go across its waves by way of
// LDS.  Bound by memory for many rows, by the chain load, sums, store for few.
// Loads and stores are of 16 bytes at any alignment; where a row is no whole chunks of eight, its
// last thread takes the last eight values and skips those of the one before it (8192 rows of 8192
// in bfloat16, both norms and a gate: 120 us, 4.5 TB/s; 8 rows of 4096 9.3 us, 5.6 of kernel; 4096 rows of 8190
// in bfloat16, both norms: 66 us, 60.5 of 8192; value by value 292).
// Values and sums are in 32 bits, in 64 with a FIELD output: its whole numbers are
// chosen next to borders and reach 2^30, beyond what 32 bits hold.
#pragma once
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

// The sum over the workgroup, the same in every thread.  `turn`: which half of `part`;
// none is written again before every thread has read it (a barrier lies between).
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

// Eight values as they lie in memory, of an element size known when it is compiled.  Which
// of the two types of a size they have is a select: branches would end every load's flight.
template <int kSize>
struct Chunk;
template <>
struct Chunk<2> {
    u32x4_ r;
    __device__ __forceinline__ void load(const void* p, size_t i) { r = *(const u32x4_at2*)((const uint16_t*)p + i); }
    template <typename A>
    __device__ __forceinline__ typename Eight<A>::V values(int type, float) const {
        typedef __bf16 B8 __attribute__((ext_vector_type(8)));
        typedef _Float16 H8 __attribute__((ext_vector_type(8)));
        const B8 b = __builtin_bit_cast(B8, r);
        const H8 h = __builtin_bit_cast(H8, r);
        typename Eight<A>::V v;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (A)(type == MVK_TYPE_BF16 ? (float)b[k] : (float)h[k]);
        return v;
    }
};
template <>
struct Chunk<4> {
    u32x4_ lo, hi;
    __device__ __forceinline__ void load(const void* p, size_t i) {
        lo = ((const u32x4_at4*)((const uint32_t*)p + i))[0];
        hi = ((const u32x4_at4*)((const uint32_t*)p + i))[1];
    }
    template <typename A>
    __device__ __forceinline__ typename Eight<A>::V values(int type, float scale) const {
        typename Eight<A>::V v;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t x = k < 4 ? lo[k & 3] : hi[k & 3];
            const A f = (A)__uint_as_float(x), y = Eight<A>::lift(x, scale);
            v[k] = type == MVK_TYPE_F32 ? f : y;
        }
        return v;
    }
};

// Eight values of a norm's parameters or a gate.
template <typename A>
__device__ __forceinline__ typename Eight<A>::V load_params(const void* p, int type, size_t i) {
    if (type == MVK_TYPE_F32) {
        Chunk<4> c;
        c.load(p, i);
        return c.values<A>(MVK_TYPE_F32, 0.f);
    }
    Chunk<2> c;
    c.load(p, i);
    return c.values<A>(type, 0.f);
}

// A norm of v, rows of n = 1 / share values (zeros for what a thread skips), by parameters as
// `params` loads them.
template <typename A, int kEach, typename Params>
__device__ __forceinline__ void apply_norm(typename Eight<A>::V (&v)[kEach], const Piece (&at)[kEach], const NormView& w, A share,
                                           A (*part)[16], uint32_t& turn, Params params) {
    if (w.kind == MVK_NORM_LAYER) {
        A sum = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) sum += v[i][k];
        const A mean = group_sum(sum, part, turn) * share;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) v[i][k] = k >= at[i].skip ? v[i][k] - mean : (A)0;
    }
    A sq = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) sq += v[i][k] * v[i][k];
    const A r = (A)1 / sqrt(group_sum(sq, part, turn) * share + (A)w.eps);
#pragma unroll
    for (int i = 0; i < kEach; ++i) v[i] *= r;
    if (w.weight) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i] *= params(w.weight, i);
    }
    if (w.bias) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i] += params(w.bias, i);
    }
}

// Rows of eight values and more, of any alignment.  kEach chunks of eight values a thread: chunk
// tid, tid + threads, ...; kX, kS: element sizes of x and of the residual.
// kWhole: rows of whole chunks (their last threads' selects and stores cost the others 4 % in any
// alignment: 8192 rows of 8192 in bfloat16, both norms and a gate, 120 us and 125).
template <typename A, int kThreads, int kEach, int kX, int kS, bool kWhole>
__global__ __launch_bounds__(kThreads) void block_norm(NormArgs a) {
    typedef typename Eight<A>::V V;
    __shared__ A part[2][16];
    uint32_t turn = 0;
    const uint32_t n = a.n;
    Piece at[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const uint32_t c = threadIdx.x + i * blockDim.x;
        at[i] = !kWhole ? piece_of(c, n) : 8 * c < n ? Piece{8 * c, 0} : Piece{0, 8};
    }
    const A share = (A)1 / (A)n;
    Chunk<kX> x[kEach];
    Chunk<kS> res[kEach];
    auto load = [&](uint32_t t) {
        if (a.x.p) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) x[i].load(a.x.p, t * a.x.stride + at[i].at);
        }
        if (a.res.p) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) res[i].load(a.res.p, t * a.res.stride + at[i].at);
        }
    };
    // zeros for what another thread has: values, and what residual and biases made of them
    auto skip = [&](V (&v)[kEach]) {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (kWhole) {
                if (at[i].skip) v[i] = V{};
            } else if (at[i].skip) {
#pragma unroll
                for (uint32_t k = 0; k < 8; ++k) v[i][k] = k >= at[i].skip ? v[i][k] : (A)0;
            }
    };
    auto store = [&](const Matrix& m, uint32_t t, const V (&v)[kEach], A inv_scale) {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (kWhole) {
                if (!at[i].skip) store8<A>(m.p, m.type, t * m.stride + at[i].at, v[i], inv_scale);
            } else if (at[i].skip < 8) {
                store_piece<A>(m.p, m.type, t * m.stride, at[i], v[i], inv_scale);
            }
    };
    if (blockIdx.x < a.T) load(blockIdx.x);
    for (uint32_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        V v[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i] = V{};
        if (a.x.p) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) v[i] = x[i].template values<A>(a.x.type, a.x_scale);
            skip(v);
            if (a.after.on)
                apply_norm<A, kEach>(v, at, a.after, share, part, turn,
                                     [&](const void* p, int i) { return load_params<A>(p, a.after.type, at[i].at); });
            if (a.gate.p) {
#pragma unroll
                for (int i = 0; i < kEach; ++i) v[i] *= load_params<A>(a.gate.p, a.gate.type, t * a.gate.stride + at[i].at);
            }
#pragma unroll
            for (int i = 0; i < kEach; ++i) v[i] *= (A)a.scale;
        }
        if (a.res.p) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) v[i] += res[i].template values<A>(a.res.type, 0.f);
        }
        // the next row's loads run behind what is left of this one
        if (t + gridDim.x < a.T) load(t + gridDim.x);
        skip(v);
        if (a.res_out.p) store(a.res_out, t, v, (A)1);
        if (!a.out.p) continue;
        if (a.before.on)
            apply_norm<A, kEach>(v, at, a.before, share, part, turn,
                                 [&](const void* p, int i) { return load_params<A>(p, a.before.type, at[i].at); });
        store(a.out, t, v, (A)1 / (A)a.out_scale);
    }
}

inline int size_of(const Matrix& m) { return m.type <= MVK_TYPE_F16 ? 2 : 4; }

template <typename A, int kX, int kS, bool kWhole>
hipError_t launch_norm_of(const NormArgs& a, hipStream_t s) {
    const uint32_t chunks = (a.n + 7) / 8;
    auto go = [&](auto kernel, uint32_t most, uint32_t each) {
        uint32_t threads = ((chunks + each - 1) / each + 63) / 64 * 64;
        threads = threads < most ? threads : most;
        // 2048 threads a compute unit, each workgroup with the next row's loads in flight (one a row:
        // 126 us where this takes 122)
        const uint32_t groups = 256 * 2048 / threads;
        hipLaunchKernelGGL(kernel, dim3(a.T < groups ? a.T : groups), dim3(threads), 0, s, a);
        return hipGetLastError();
    };
    // Few rows: as many threads as the row can use.  Many: two chunks a thread.  Kernels of both norms in
    // bfloat16, us, by one chunk and by two: 8 rows of 4096 4.8 and 5.7, 256 of 4097 6.7 and 7.4, 512 of
    // 4096 7.1 and 7.5; the same at 64 rows of 8192 (6.1 and 6.0), but 512 11.6 and 9.9, 8192 161 and 126
    // (by four chunks 156).
    if (chunks <= 256) return go(block_norm<A, 256, 1, kX, kS, kWhole>, 256, 1);
    if (chunks <= 1024 && a.T <= 512) return go(block_norm<A, 1024, 1, kX, kS, kWhole>, 1024, 1);
    if (chunks <= 512) return go(block_norm<A, 256, 2, kX, kS, kWhole>, 256, 2);
    if (chunks <= 1024) return go(block_norm<A, 512, 2, kX, kS, kWhole>, 512, 2);
    if (chunks <= 2048) return go(block_norm<A, 1024, 2, kX, kS, kWhole>, 1024, 2);
    return go(block_norm<A, 1024, 4, kX, kS, kWhole>, 1024, 4);
}

// By the sizes of x's and the residual's values.
template <typename A, bool kWhole>
hipError_t launch_norm_in(const NormArgs& a, hipStream_t s) {
    const int kx = a.x.p ? size_of(a.x) : 4, ks = a.res.p ? size_of(a.res) : 4;
    if (kx == 2) return ks == 2 ? launch_norm_of<A, 2, 2, kWhole>(a, s) : launch_norm_of<A, 2, 4, kWhole>(a, s);
    return ks == 2 ? launch_norm_of<A, 4, 2, kWhole>(a, s) : launch_norm_of<A, 4, 4, kWhole>(a, s);
}

}  // namespace

}  // namespace mvk
