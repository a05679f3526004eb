// Rows of values of a type known at run time, eight consecutive ones at once.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "kv.h"

namespace mvk {

// A matrix: element i of row t at p[t * stride + i]; wide: every row is made of whole
// aligned 16-byte granules, as far as whole eights of its values go.
struct Matrix {
    void* p;
    size_t stride;
    int type;
    bool wide;
};

inline bool is_wide(const void* p, size_t stride, int type, uint64_t rows) {
    const size_t per = type == MVK_TYPE_BF16 || type == MVK_TYPE_F16 ? 8 : 4;
    return (uintptr_t)p % 16 == 0 && (rows <= 1 || stride % per == 0);
}

// A norm's parameters; on: there is one.
struct NormView {
    const void *weight, *bias;
    int type, kind;
    float eps;
    bool wide, on;
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
    float in_scale, inv_scale;
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
        r.lo = *(const u32x4_*)((const uint16_t*)p + i);
        r.hi = r.lo;
    } else {
        r.lo = ((const u32x4_*)((const uint32_t*)p + i))[0];
        r.hi = ((const u32x4_*)((const uint32_t*)p + i))[1];
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

// Values i .. i + 7 (count of them; the others are zero).
template <typename A>
__device__ __forceinline__ typename Eight<A>::V load8(const void* p, int type, bool wide, size_t i, uint32_t count, float scale) {
    if (wide && count >= 8) return values_of<A>(load_raw8(p, type, i), type, scale);
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

template <typename A>
__device__ __forceinline__ void store8(void* p, int type, bool wide, size_t i, uint32_t count, typename Eight<A>::V v, A inv_scale) {
    if (wide && count >= 8) {
        if (type == MVK_TYPE_BF16) {
            typedef __bf16 B8 __attribute__((ext_vector_type(8)));
            B8 x;
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = (__bf16)(float)v[k];
            *(u32x4_*)((uint16_t*)p + i) = __builtin_bit_cast(u32x4_, x);
        } else if (type == MVK_TYPE_F16) {
            typedef _Float16 H8 __attribute__((ext_vector_type(8)));
            H8 x;
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = (_Float16)(float)v[k];
            *(u32x4_*)((uint16_t*)p + i) = __builtin_bit_cast(u32x4_, x);
        } else {
            const bool field = type == MVK_TYPE_FIELD;
            u32x4_ lo, hi;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                lo[k] = field ? field_of(v[k] * inv_scale) : __float_as_uint((float)v[k]);
                hi[k] = field ? field_of(v[k + 4] * inv_scale) : __float_as_uint((float)v[k + 4]);
            }
            ((u32x4_*)((uint32_t*)p + i))[0] = lo;
            ((u32x4_*)((uint32_t*)p + i))[1] = hi;
        }
        return;
    }
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) {
        if (k >= count) break;
        if (type == MVK_TYPE_BF16) ((__bf16*)p)[i + k] = (__bf16)(float)v[k];
        else if (type == MVK_TYPE_F16) ((_Float16*)p)[i + k] = (_Float16)(float)v[k];
        else if (type == MVK_TYPE_F32) ((float*)p)[i + k] = (float)v[k];
        else ((uint32_t*)p)[i + k] = field_of(v[k] * inv_scale);
    }
}

}  // namespace mvk
