// The gated activation: out = act(gate) * up, value by value, in 32 bits.  One pass,
// bound by memory.
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

// A thread eight values of a row, in loads of 16 bytes at any alignment.  (A value by value form for
// rows that are no whole granules took 154 us for 4096 rows of 11007 in bfloat16; 58 those of 11008.)
__global__ __launch_bounds__(256) void gated_activation(GatedArgs a, uint32_t chunks, uint64_t count) {
    for (uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x; id < count; id += (uint64_t)gridDim.x * 256) {
        const uint32_t t = (uint32_t)(id / chunks);
        const size_t g0 = t * a.gate.stride, u0 = t * a.up.stride, o0 = t * a.out.stride;
        f32x8 g, u;
        if (a.n < 8) {
            g = load_some<float>(a.gate.p, a.gate.type, g0, a.n, a.in_scale);
            u = load_some<float>(a.up.p, a.up.type, u0, a.n, a.in_scale);
        }
        const Piece p = a.n < 8 ? Piece{0, 8 - a.n} : piece_of((uint32_t)(id % chunks), a.n);
        if (a.n >= 8) {
            g = values_of<float>(load_raw8(a.gate.p, a.gate.type, g0 + p.at), a.gate.type, a.in_scale);
            u = values_of<float>(load_raw8(a.up.p, a.up.type, u0 + p.at), a.up.type, a.in_scale);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) g[k] = activate(g[k], a.act) * u[k];
        if (a.n < 8) store_some<float>(a.out.p, a.out.type, o0, 0, a.n, g, a.inv_scale);
        else store_piece<float>(a.out.p, a.out.type, o0, p, g, a.inv_scale);
    }
}

}  // namespace

hipError_t launch_gated(const GatedArgs& a, hipStream_t s) {
    const uint32_t chunks = (uint32_t)(((uint64_t)a.n + 7) / 8);
    const uint64_t count = (uint64_t)a.T * chunks, blocks = (count + 255) / 256;
    hipLaunchKernelGGL(gated_activation, dim3((uint32_t)(blocks < (1u << 22) ? blocks : 1u << 22)), dim3(256), 0, s, a,
                       chunks, count);
    return hipGetLastError();
}

}  // namespace mvk
