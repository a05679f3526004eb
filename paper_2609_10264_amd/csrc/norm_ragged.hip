// block_norm (norm.h) of rows that are no whole chunks of eight values.
#include "norm.h"

namespace mvk {

namespace {

// Rows of fewer than eight values: one thread's.
template <typename A>
__global__ __launch_bounds__(64) void block_norm_short(NormArgs a) {
    typedef typename Eight<A>::V V;
    __shared__ A part[2][16];  // (not used: one wave)
    uint32_t turn = 0;
    // (as a piece: the values are the last ones of the eight)
    const uint32_t n = threadIdx.x == 0 ? a.n : 0;
    const Piece at[1] = {{0, 8 - n}};
    const A share = (A)1 / (A)a.n;
    auto load = [&](const void* p, int type, size_t row, float scale) {
        V v;
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) v[k] = k >= 8 - n ? load_one<A>(p, type, row + k - (8 - n), scale) : (A)0;
        return v;
    };
    auto store = [&](const Matrix& m, size_t row, V v, A inv_scale) {
        V first = {};
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k)
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) first[j] = k >= 8 - n && k - (8 - n) == j ? v[k] : first[j];
        store_some<A>(m.p, m.type, row, 0, n, first, inv_scale);
    };
    for (uint32_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        V v[1] = {};
        if (a.x.p) {
            v[0] = load(a.x.p, a.x.type, t * a.x.stride, a.x_scale);
            if (a.after.on)
                apply_norm<A, 1>(v, at, a.after, share, part, turn, [&](const void* p, int) { return load(p, a.after.type, 0, 0.f); });
            if (a.gate.p) v[0] *= load(a.gate.p, a.gate.type, t * a.gate.stride, 0.f);
            v[0] *= (A)a.scale;
        }
        if (a.res.p) v[0] += load(a.res.p, a.res.type, t * a.res.stride, 0.f);
        if (a.res_out.p) store(a.res_out, t * a.res_out.stride, v[0], (A)1);
        if (!a.out.p) continue;
        if (a.before.on)
            apply_norm<A, 1>(v, at, a.before, share, part, turn, [&](const void* p, int) { return load(p, a.before.type, 0, 0.f); });
        store(a.out, t * a.out.stride, v[0], (A)1 / (A)a.out_scale);
    }
}

template <typename A>
hipError_t launch_ragged(const NormArgs& a, hipStream_t s) {
    if (a.n >= 8) return launch_norm_in<A, false>(a, s);
    hipLaunchKernelGGL(block_norm_short<A>, dim3(a.T < (1u << 20) ? a.T : 1u << 20), dim3(64), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_block_norm_ragged(const NormArgs& a, hipStream_t s) {
    return a.out.p && a.out.type == MVK_TYPE_FIELD ? launch_ragged<double>(a, s) : launch_ragged<float>(a, s);
}

}  // namespace mvk
