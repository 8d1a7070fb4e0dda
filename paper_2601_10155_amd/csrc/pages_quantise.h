// The pages' 8-bit rounding: exponents, stored bytes, a token's codes.
#pragma once

#include "pages.h"

namespace lookat {

typedef float v2f __attribute__((ext_vector_type(2)));

template <bool FP8>
__device__ __forceinline__ int exponent_of(float top)
{
    const uint32_t bits = __float_as_uint(top);
    const int e = (int)(bits >> 23) - 127;
    const uint32_t mant = bits & 0x7fffffu;
    // largest stored number: 127 = 1.984375 * 2^6, 448 = 1.75 * 2^8
    const int x = FP8 ? e - 8 + (mant > 0x600000u) : e - 6 + (mant > 0x7e0000u);
    return x < kLowExponent ? kLowExponent : x > kHighExponent ? kHighExponent : x;   // (zero and fp32's subnormals: the lowest)
}
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // e in [-126, 127]

// Four scaled numbers to four stored bytes.
template <bool FP8>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d)
{
    constexpr float top = FP8 ? 448.f : 127.f;
    const float x[4] = {a, b, c, d};
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float r = FP8 ? x[i] : rintf(x[i]);
        y[i] = r != r ? 0.f : fminf(fmaxf(r, -top), top);
    }
    if constexpr (FP8) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    } else {
        return ((uint32_t)(int)y[0] & 0xffu) | ((uint32_t)(int)y[1] & 0xffu) << 8 | ((uint32_t)(int)y[2] & 0xffu) << 16 |
               (uint32_t)(int)y[3] << 24;
    }
}
template <bool FP8>
__device__ __forceinline__ void unpack4(uint32_t w, float (&x)[4])
{
    if constexpr (FP8) {
        const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        x[0] = lo.x, x[1] = lo.y, x[2] = hi.x, x[3] = hi.y;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[i] = (float)(int8_t)(w >> (8 * i));
    }
}

// An exponent that these kernels did not write may be any int8: 2^(old - e) is then below 2^-126, whose products round to zero too.
__device__ __forceinline__ float rescale(int old_e, int e) { return two_to(old_e - e < -126 ? -126 : old_e - e); }

// codes of one token, m bytes, aligned to m
__device__ __forceinline__ void copy_code(uint8_t *dst, const uint8_t *src, int m, int t)
{
    if (m == 2)
        reinterpret_cast<uint16_t *>(dst)[t] = reinterpret_cast<const uint16_t *>(src)[t];
    else if (m == 4)
        reinterpret_cast<uint32_t *>(dst)[t] = reinterpret_cast<const uint32_t *>(src)[t];
    else if (m == 8)
        reinterpret_cast<uint2 *>(dst)[t] = reinterpret_cast<const uint2 *>(src)[t];
    else
        reinterpret_cast<u32x4 *>(dst)[t] = reinterpret_cast<const u32x4 *>(src)[t];
}

}  // namespace lookat
