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

// A thread eight values of a row.
__global__ __launch_bounds__(256) void gated_activation(GatedArgs a, uint32_t chunks, uint64_t count) {
    for (uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x; id < count; id += (uint64_t)gridDim.x * 256) {
        const uint32_t t = (uint32_t)(id / chunks), at = 8 * (uint32_t)(id % chunks), c = min(8u, a.n - at);
        f32x8 g = load8<float>(a.gate.p, a.gate.type, a.gate.wide, t * a.gate.stride + at, c, a.in_scale);
        const f32x8 u = load8<float>(a.up.p, a.up.type, a.up.wide, t * a.up.stride + at, c, a.in_scale);
#pragma unroll
        for (int k = 0; k < 8; ++k) g[k] = activate(g[k], a.act) * u[k];
        store8<float>(a.out.p, a.out.type, a.out.wide, t * a.out.stride + at, c, g, a.inv_scale);
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
