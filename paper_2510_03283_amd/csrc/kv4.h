// The 4-bit values of the paged cache (gfx950): sign, two bits of exponent, one of mantissa (magnitudes 0, 1/2, 1, 3/2, 2, 3, 4, 6), two a byte, the
// even element in the low half, and for 32 neighbours of a head one byte b that stands for 2^(b - 127), 255 for NaN.
#pragma once
#include "common.h"

namespace kv4 {

constexpr int GROUP = 32;              // values that share a scale
constexpr uint32_t NAN_SCALE = 255;

// Scale byte of a group from the bits of its largest magnitude: 2^(floor(log2 top) - 2), twice that where top is above 7 steps, so that no value
// is off by more than half of its own step (the step at 6 being 2).  Limits 3 and 252: every value is then a normal number of bf16 and below infinity.
// Of normally distributed values the error is 0.1119 of their norm; without the 7 (top up to 8 steps, cut to 6) 0.1150, without any cut 0.1155.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top_bits) {
  if (top_bits >= 0x7f800000u) return NAN_SCALE;
  const int b = (int)(top_bits >> 23) - 2 + ((top_bits & 0x7fffffu) > 0x600000u);
  return (uint32_t)min(max(b, 3), 252);
}
// (byte 0 would be the subnormal 2^-127; the conversions take the exponent field alone)
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight fp32 values -> eight codes, nearest, ties to even, at most 6 steps.
__device__ __forceinline__ uint32_t encode8(const float (&x)[8], float scale) {
  uint32_t u = 0;
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[0], x[1], scale, 0);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[2], x[3], scale, 1);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[4], x[5], scale, 2);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[6], x[7], scale, 3);
  return u;
}
// Eight codes -> eight bf16 values, exact.
__device__ __forceinline__ bf16x8_t decode8(uint32_t u, float scale) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 0));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 1));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 2));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 3));
  return __builtin_bit_cast(bf16x8_t, r);
}

}  // namespace kv4
