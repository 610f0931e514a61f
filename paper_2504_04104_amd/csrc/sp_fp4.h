// Values held in 4 bits (e2m1: sign, two exponent bits, one mantissa bit) with one power of two for 32 of them.
//
// A group's scale is 2^e for the smallest e in [-100, 125] with max |x| <= 6 * 2^e, stored as e + 127; a value is
// +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} * 2^e, rounded to nearest with ties to the even code: off by at most 2^e, half of the widest gap,
// where the group's largest value is above 3 * 2^e (or e is -100).  All of it is exact in bfloat16 (e >= -100 keeps the smallest
// value normal, e <= 125 the largest finite), so a product of held values takes the bf16 matrix instructions without another
// rounding.  What 4 bits cannot hold: an infinity is held as +-6 * 2^125, a NaN as zero; what is read back is always finite.
#pragma once
#include "sp_device.h"

#define FP4_GROUP 32

// The scale as a float whose exponent field is the stored byte (a byte of zero: cleared storage, whose codes are zeros too).
__device__ __forceinline__ float fp4_scale(uint32_t biased) { return __uint_as_float(biased << 23); }

// Eight codes, lowest bits first, as a bf16 matrix operand.  (The conversion takes the exponent field of the scale and nothing
// else of it.)
__device__ __forceinline__ u32x4_t fp4_to_bf16x8(uint32_t codes, float scale) {
  return (u32x4_t){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}

// The stored scale of a group whose largest magnitude is amax: 1.5 * 2^(e + 2) is the largest value.
__device__ __forceinline__ uint32_t fp4_biased(float amax) {
  const uint32_t bits = __float_as_uint(amax) & 0x7fffffffu;
  const int b = (int)(bits >> 23) - 2 + ((bits & 0x7fffffu) > 0x400000u ? 1 : 0);
  return (uint32_t)min(max(b, 27), 252);
}
__device__ __forceinline__ float fp4_clean(float x) { return x == x ? x : 0.f; }
// Four values of a group as 16 bits of codes.
__device__ __forceinline__ uint32_t fp4_codes4(const float (&v)[4], float scale) {
  const uint32_t lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, fp4_clean(v[0]), fp4_clean(v[1]), scale, 0);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(lo, fp4_clean(v[2]), fp4_clean(v[3]), scale, 1) & 0xffffu;
}
