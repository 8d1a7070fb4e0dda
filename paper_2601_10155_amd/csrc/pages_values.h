// Stored 8-bit values as operands of the matrix cores, and the running reference of a softmax whose logits carry the pages' exponents: what
// attention of one token and of a chunk over the pages share.
#pragma once

#include "pages.h"
#include "decode_common.h"

namespace lookat {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

constexpr float kRefLag = 8.f;            // the reference moves when a logit exceeds it by more (log2 units)
constexpr float kNoReference = -3.402823466e38f;   // before the first token: fp32's lowest, so no logit is below it, and finite: -inf less it is -inf
constexpr float kRefLift = 7.f;           // weights are 2^7 at the reference, below 2^15: fp16's range, its subnormals far below

// Eight stored bytes (two registers) to eight fp16 numbers, exactly.
template <bool FP8>
__device__ __forceinline__ v8h widen(uint32_t lo, uint32_t hi)
{
    uint32_t w[4];
    if constexpr (FP8) {
        const v2h a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
        const v2h c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
        w[0] = __builtin_bit_cast(uint32_t, a);
        w[1] = __builtin_bit_cast(uint32_t, b);
        w[2] = __builtin_bit_cast(uint32_t, c);
        w[3] = __builtin_bit_cast(uint32_t, d);
    } else {
        // q + 128 behind the exponent byte of 1024: 1024 + 128 + q, less 1152
        const v2h bias = {(_Float16)-1152.f, (_Float16)-1152.f};
        lo ^= 0x80808080u;
        hi ^= 0x80808080u;
        const uint32_t u[4] = {__builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u),
                               __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u)};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = __builtin_bit_cast(uint32_t, (v2h)(__builtin_bit_cast(v2h, u[i]) + bias));
    }
    const v4u r = {w[0], w[1], w[2], w[3]};
    return __builtin_bit_cast(v8h, r);
}

}  // namespace lookat
