// Values held in 8 bits with a power of two for a row: code * 2^e.
//
// e is the least exponent in range with max |x| <= M 2^e (M: the largest code), so
// x / 2^e is exact and a code is one rounding of x.  Both formats then are exact in
// bfloat16 (4 and 7 significant bits).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kv.h"

namespace mvk {

// How the values of a cache of type T are held (S), what attention computes with
// (Q), and their value (`two`: of power()).
template <typename T>
struct Held {
    typedef T Q;
    typedef T S;
    static constexpr bool k8 = false;
    static __device__ __forceinline__ float get(S x, float) { return to_float(x); }
};
struct E4M3 {};
struct I8 {};
template <>
struct Held<E4M3> {
    typedef __bf16 Q;
    typedef uint8_t S;
    static constexpr bool k8 = true;
    static constexpr int kBits = 8;               // M = 1.75 2^8
    static constexpr uint32_t kMantissa = 0xc0000u;  // of M, the first 20 bits (the others are zero)
    static constexpr float kMost = 448.f;
    static __device__ __forceinline__ float get(S x, float two) { return __builtin_amdgcn_cvt_f32_fp8((int)x, 0) * two; }
    // Two codes of y, z within M (the conversion rounds to nearest, ties to even).
    static __device__ __forceinline__ uint32_t codes(float y, float z) {
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y, z, 0, false) & 0xffffu;
    }
};
template <>
struct Held<I8> {
    typedef __bf16 Q;
    typedef uint8_t S;
    static constexpr bool k8 = true;
    static constexpr int kBits = 6;               // M = 1.984375 2^6
    static constexpr uint32_t kMantissa = 0xfc000u;
    static constexpr float kMost = 127.f;
    static __device__ __forceinline__ float get(S x, float two) { return (float)(int8_t)x * two; }
    static __device__ __forceinline__ uint32_t codes(float y, float z) {
        return ((uint32_t)(int32_t)rintf(y) & 0xffu) | ((uint32_t)(int32_t)rintf(z) & 0xffu) << 8;
    }
};

// 2^e of an exponent in range; a not-a-number of MVK_EXP_NAN.
__device__ __forceinline__ float power(int e) {
    return __uint_as_float(e == MVK_EXP_NAN ? 0x7fc00000u : (uint32_t)(e + 127) << 23);
}

// Eight consecutive values in bfloat16, exactly (of a value: codes of one byte, the first lowest).
typedef uint32_t u32x2_ __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4q __attribute__((ext_vector_type(4)));
template <typename C>
__device__ __forceinline__ u32x4q widen(u32x2_ codes, float two) {
    u32x4q y;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        if (__is_same(C, E4M3)) {
            y[2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[w], two, false));
            y[2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[w], two, true));
        } else {
            // from 128 on, as bytes convert in one instruction: (u - 128) two, without a rounding
            typedef float F2 __attribute__((ext_vector_type(2)));
            typedef __bf16 B2 __attribute__((ext_vector_type(2)));
            const uint32_t u = codes[w] ^ 0x80808080u;
            const float low = -128.f * two;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const F2 f = {__builtin_fmaf((float)(u >> (16 * h) & 0xffu), two, low),
                              __builtin_fmaf((float)(u >> (16 * h + 8) & 0xffu), two, low)};
                y[2 * w + h] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, B2));
            }
        }
    }
    return y;
}

// The first 32 bits of |x|, the last of them set where later ones are: orders as |x|
// does against any value whose later bits are zero.  0 of infinities and not-a-numbers.
__device__ __forceinline__ uint32_t top_bits(double x) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t hi = (uint32_t)(b >> 32) & 0x7fffffffu;
    return hi >= 0x7ff00000u ? 0u : hi | ((uint32_t)b != 0 ? 1u : 0u);
}
// (of a float, as of the double it is)
__device__ __forceinline__ uint32_t top_bits(float x) { return top_bits((double)x); }
__device__ __forceinline__ bool is_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }
__device__ __forceinline__ bool is_finite(double x) {
    return ((uint32_t)(__builtin_bit_cast(uint64_t, x) >> 32) & 0x7ff00000u) != 0x7ff00000u;
}

// The exponent of a row whose largest top_bits is `top`.
template <typename C>
__device__ __forceinline__ int row_exponent(uint32_t top) {
    const int e = (int)(top >> 20) - 1023 - Held<C>::kBits + ((top & 0xfffffu) > Held<C>::kMantissa ? 1 : 0);
    return max(MVK_EXP_LEAST, min(MVK_EXP_MOST, e));
}

// x / 2^e within M, rounded to 32 bits so that a later rounding to few bits gives what
// rounding x itself would (towards zero, the last bit set where something was lost).
template <typename C>
__device__ __forceinline__ float scaled(double x, int e) {
    const double y = x * __builtin_bit_cast(double, (uint64_t)(1023 - e) << 52);
    const float f = (float)y;
    const double d = (double)f;
    uint32_t b = __float_as_uint(f);
    if (d != y) b = (fabs(d) > fabs(y) ? b - 1 : b) | 1u;
    return __builtin_amdgcn_fmed3f(__uint_as_float(b), -Held<C>::kMost, Held<C>::kMost);
}
// The same of a float, which is exact but where the code is zero anyway.
template <typename C>
__device__ __forceinline__ float scaled(float x, int e) {
    return __builtin_amdgcn_fmed3f(x * __uint_as_float((uint32_t)(127 - e) << 23), -Held<C>::kMost, Held<C>::kMost);
}

// A field element or a float in 64 bits (a 31-bit residue times a power of two is exact).
__device__ __forceinline__ double to_double(float x) { return (double)x; }
__device__ __forceinline__ double to_double(__bf16 x) { return (double)(float)x; }
__device__ __forceinline__ double to_double(_Float16 x) { return (double)(float)x; }
__device__ __forceinline__ int32_t field_centred(uint32_t y) { return y > kP / 2 ? (int32_t)(y - kP) : (int32_t)y; }

}  // namespace mvk
