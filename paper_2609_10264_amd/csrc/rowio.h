// Rows of values of a type known at run time, eight consecutive ones at once.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "kv.h"

namespace mvk {

// A matrix: element i of row t at p[t * stride + i].
struct Matrix {
    void* p;
    size_t stride;
    int type;
};

// A norm's parameters; on: there is one.
struct NormView {
    const void *weight, *bias;
    int type, kind;
    float eps;
    bool on;
};

// Of block_norm (norm.hip), gated_activation (gated.hip), sample_tokens (draw.hip);
// matrices without data are not there.
struct NormArgs {
    Matrix x, res, gate, res_out, out;
    NormView after, before;
    uint32_t T, n;
    float x_scale, scale, out_scale;
};
struct GatedArgs {
    Matrix gate, up, out;
    uint32_t T, n;
    int act;
    float in_scale, out_scale;
};
struct DrawArgs {
    Matrix x;
    uint32_t R, n;
    float scale;  // of FIELD logits
    mvk_sampling how;
    const float* u;
    int32_t* tokens;
    float* probs;
};

typedef uint32_t u32x4_ __attribute__((ext_vector_type(4)));
// (of any place of a row: memory takes 16 bytes at once whatever their alignment is)
typedef uint32_t u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef double f64x8 __attribute__((ext_vector_type(8)));
template <typename A>
struct Eight;
template <>
struct Eight<float> {
    typedef f32x8 V;
    static __device__ __forceinline__ float lift(uint32_t y, float scale) { return field_lift(y) * scale; }
};
template <>
struct Eight<double> {
    typedef f64x8 V;
    static __device__ __forceinline__ double lift(uint32_t y, float scale) {
        return (double)(y > kP / 2 ? (int32_t)(y - kP) : (int32_t)y) * (double)scale;
    }
};

// Element i alone.
template <typename A>
__device__ __forceinline__ A load_one(const void* p, int type, size_t i, float scale) {
    if (type == MVK_TYPE_BF16) return (A)(float)((const __bf16*)p)[i];
    if (type == MVK_TYPE_F16) return (A)(float)((const _Float16*)p)[i];
    if (type == MVK_TYPE_F32) return (A)((const float*)p)[i];
    return Eight<A>::lift(((const uint32_t*)p)[i], scale);
}

// Eight values from element i on, as they lie in memory (16 or 32 bytes).
struct Raw8 {
    u32x4_ lo, hi;
};
__device__ __forceinline__ Raw8 load_raw8(const void* p, int type, size_t i) {
    Raw8 r;
    if (type <= MVK_TYPE_F16) {
        r.lo = *(const u32x4_at2*)((const uint16_t*)p + i);
        r.hi = r.lo;
    } else {
        r.lo = ((const u32x4_at4*)((const uint32_t*)p + i))[0];
        r.hi = ((const u32x4_at4*)((const uint32_t*)p + i))[1];
    }
    return r;
}
template <typename A>
__device__ __forceinline__ typename Eight<A>::V values_of(const Raw8& r, int type, float scale) {
    typename Eight<A>::V v;
    if (type == MVK_TYPE_BF16) {
        typedef __bf16 B8 __attribute__((ext_vector_type(8)));
        const B8 x = __builtin_bit_cast(B8, r.lo);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (A)(float)x[k];
    } else if (type == MVK_TYPE_F16) {
        typedef _Float16 H8 __attribute__((ext_vector_type(8)));
        const H8 x = __builtin_bit_cast(H8, r.lo);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (A)(float)x[k];
    } else if (type == MVK_TYPE_F32) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (A)__uint_as_float(r.lo[k]), v[k + 4] = (A)__uint_as_float(r.hi[k]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = Eight<A>::lift(r.lo[k], scale), v[k + 4] = Eight<A>::lift(r.hi[k], scale);
    }
    return v;
}

// Eight consecutive values of a row of n >= 8 by one thread: chunk c, or, where the row ends
// within it, the row's last eight, of which the first `skip` are the chunk before's (8: all).
struct Piece {
    uint32_t at, skip;
};
__device__ __forceinline__ Piece piece_of(uint32_t c, uint32_t n) {
    const uint32_t at = 8 * c;
    if (at + 8 <= n) return {at, 0u};
    return at < n ? Piece{n - 8, at + 8 - n} : Piece{0u, 8u};
}

// Values i .. i + count - 1 one by one; the others are zero.
template <typename A>
__device__ __forceinline__ typename Eight<A>::V load_some(const void* p, int type, size_t i, uint32_t count, float scale) {
    typename Eight<A>::V v;
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) v[k] = k < count ? load_one<A>(p, type, i + k, scale) : (A)0;
    return v;
}

// The field element of the integer nearest to x, in 64 bits (as field_of in 32).
__device__ __forceinline__ uint32_t field_of(double x) {
    constexpr double half = (double)((kP - 1) / 2);
    const double r = fmin(fmax(x == x ? rint(x) : 0., -half), half);
    const int32_t i = (int32_t)r;
    return i < 0 ? kP + (uint32_t)i : (uint32_t)i;
}

// (64 bits to 16 in one rounding, not by way of 32)
template <typename A>
__device__ __forceinline__ void store8(void* p, int type, size_t i, typename Eight<A>::V v, A inv_scale) {
    if (type == MVK_TYPE_BF16) {
        typedef __bf16 B8 __attribute__((ext_vector_type(8)));
        B8 x;
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = (__bf16)v[k];
        *(u32x4_at2*)((uint16_t*)p + i) = __builtin_bit_cast(u32x4_, x);
    } else if (type == MVK_TYPE_F16) {
        typedef _Float16 H8 __attribute__((ext_vector_type(8)));
        H8 x;
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = (_Float16)v[k];
        *(u32x4_at2*)((uint16_t*)p + i) = __builtin_bit_cast(u32x4_, x);
    } else {
        const bool field = type == MVK_TYPE_FIELD;
        u32x4_ lo, hi;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            lo[k] = field ? field_of(v[k] * inv_scale) : __float_as_uint((float)v[k]);
            hi[k] = field ? field_of(v[k + 4] * inv_scale) : __float_as_uint((float)v[k + 4]);
        }
        ((u32x4_at4*)((uint32_t*)p + i))[0] = lo;
        ((u32x4_at4*)((uint32_t*)p + i))[1] = hi;
    }
}

// Values [from, to) of them one by one.
template <typename A>
__device__ __forceinline__ void store_some(void* p, int type, size_t i, uint32_t from, uint32_t to, typename Eight<A>::V v, A inv_scale) {
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) {
        if (k < from || k >= to) continue;
        if (type == MVK_TYPE_BF16) ((__bf16*)p)[i + k] = (__bf16)v[k];
        else if (type == MVK_TYPE_F16) ((_Float16*)p)[i + k] = (_Float16)v[k];
        else if (type == MVK_TYPE_F32) ((float*)p)[i + k] = (float)v[k];
        else ((uint32_t*)p)[i + k] = field_of(v[k] * inv_scale);
    }
}

// What a thread has of a piece.
template <typename A>
__device__ __forceinline__ void store_piece(void* p, int type, size_t row, const Piece& at, typename Eight<A>::V v, A inv_scale) {
    if (at.skip == 0) store8<A>(p, type, row + at.at, v, inv_scale);
    else store_some<A>(p, type, row + at.at, at.skip, 8, v, inv_scale);
}

}  // namespace mvk
