// The gated activation: out = act(gate) * up, value by value, in 32 bits.  One pass,
// bound by memory (8192 x 11008 in bfloat16 104 us, 5.2 TB/s; 8 rows 7 us, most of it the call).
#include "mvk_internal.h"
#include "rowio.h"

namespace mvk {

namespace {

__device__ __forceinline__ float activate(float x, int act) {
    if (act == MVK_ACT_SILU) return x / (1.f + expf(-x));
    if (act == MVK_ACT_GELU) return 0.5f * x * erfcf(x * -0.70710678118654752440f);
    if (act == MVK_ACT_GELU_TANH) {
        // (1 + tanh y) / 2 = 1 / (1 + exp(-2 y))
        const float y = 0.79788456080286535588f * (x + 0.044715f * x * x * x);
        return x / (1.f + expf(-2.f * y));
    }
    return x > 0.f || x != x ? x : 0.f;
}

// A thread eight values of a row, in loads of 16 bytes at any alignment.  kWhole: rows of whole eights
// (8192 x 11008 in bfloat16: 104 us, 110 by the other form, whose few instructions more count beside the
// activation's).  4096 rows of 11007: 59 us; value by value 154.
// A: double with a FIELD output.  Its scale is any positive number, also one whose reciprocal 32 bits
// do not hold, so the value is taken over it in 64 bits and rounded once more only, to the whole number
// (4096 x 11008, FIELD to FIELD: silu 97 us, 5.6 TB/s, gelu 101).  The value itself stays in 32 bits as
// with every output, off by (16 + 6 |g|) 2^-24 of its size at most (gelu: g^2): in 64 it takes 140 and 217.
template <typename A, bool kWhole>
__global__ __launch_bounds__(256) void gated_activation(GatedArgs a, uint32_t chunks, uint64_t count) {
    const A inv_scale = sizeof(A) == 8 ? (A)1 / (A)a.out_scale : (A)1;
    for (uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x; id < count; id += (uint64_t)gridDim.x * 256) {
        const uint32_t t = (uint32_t)(id / chunks), c = (uint32_t)(id % chunks);
        const size_t g0 = t * a.gate.stride, u0 = t * a.up.stride, o0 = t * a.out.stride;
        const Piece p = kWhole ? Piece{8 * c, 0} : a.n < 8 ? Piece{0, 0} : piece_of(c, a.n);
        f32x8 g, u;
        if (!kWhole && a.n < 8) {
            g = load_some<float>(a.gate.p, a.gate.type, g0, a.n, a.in_scale);
            u = load_some<float>(a.up.p, a.up.type, u0, a.n, a.in_scale);
        } else {
            g = values_of<float>(load_raw8(a.gate.p, a.gate.type, g0 + p.at), a.gate.type, a.in_scale);
            u = values_of<float>(load_raw8(a.up.p, a.up.type, u0 + p.at), a.up.type, a.in_scale);
        }
        typename Eight<A>::V y;
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = (A)(activate(g[k], a.act) * u[k]);
        if (!kWhole && a.n < 8) store_some<A>(a.out.p, a.out.type, o0, 0, a.n, y, inv_scale);
        else if (kWhole) store8<A>(a.out.p, a.out.type, o0 + p.at, y, inv_scale);
        else store_piece<A>(a.out.p, a.out.type, o0, p, y, inv_scale);
    }
}

}  // namespace

hipError_t launch_gated(const GatedArgs& a, hipStream_t s) {
    const uint32_t chunks = (uint32_t)(((uint64_t)a.n + 7) / 8);
    const uint64_t count = (uint64_t)a.T * chunks, blocks = (count + 255) / 256;
    const dim3 grid((uint32_t)(blocks < (1u << 22) ? blocks : 1u << 22));
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, chunks, count);
        return hipGetLastError();
    };
    if (a.out.type == MVK_TYPE_FIELD) return a.n % 8 == 0 ? go(gated_activation<double, true>) : go(gated_activation<double, false>);
    return a.n % 8 == 0 ? go(gated_activation<float, true>) : go(gated_activation<float, false>);
}

}  // namespace mvk
