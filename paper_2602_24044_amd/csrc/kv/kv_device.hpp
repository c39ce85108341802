// Device helpers of the cache in four bits: the conversions between bf16, fp32 and four-bit codes.
//
// Four bits are the e2m1 format (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) with a power of two for every 32 values, because the
// vector unit converts two of them at a time with that power applied (v_cvt_scalef32_pk_bf16_fp4, which looks at the exponent of
// its scale operand only), and because the product with a power of two is exact: a code as bf16 is the value it stands for.
#pragma once

#include "../device_common.hpp"
#include "kv_internal.hpp"

namespace lora {
namespace kv {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

// Two codes of a dword's byte SEL as bf16, times the power of two in bits 30..23 of `scale` (its other bits do not count).
template <int SEL> __device__ inline uint32_t two_bf16(uint32_t codes, uint32_t scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, __builtin_bit_cast(float, scale), SEL));
}
// The eight codes of a dword as bf16.
__device__ inline u32x4 eight_bf16(uint32_t codes, uint32_t scale)
{
    return u32x4{two_bf16<0>(codes, scale), two_bf16<1>(codes, scale), two_bf16<2>(codes, scale), two_bf16<3>(codes, scale)};
}
// Eight values as codes of a dword: divided by the power of two `scale`, rounded to the nearest code (ties to the even one), at
// most 6.
__device__ inline uint32_t eight_codes(const float (&x)[8], float scale)
{
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
    return c;
}
// Biased exponent of a group whose largest magnitude is `top`: the smallest e with top <= 7 * 2^e, where the half step behind the
// code 6 ends.  top = m 2^k with m in [1, 2), so e is k - 2 for m <= 1.75 and k - 1 above.
__device__ inline int group_exponent(float top)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, top);
    const int e = (int)(b >> 23) - 127 - ((b & 0x7fffffu) <= 0x600000u ? 2 : 1);
    return min(max(e, kMinExp), kMaxExp) + 127;
}

__device__ inline float lo_f32(uint32_t two) { return __builtin_bit_cast(float, two << 16); }
__device__ inline float hi_f32(uint32_t two) { return __builtin_bit_cast(float, two & 0xffff0000u); }
__device__ inline uint32_t pack_bf16(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

}  // namespace kv
}  // namespace lora
