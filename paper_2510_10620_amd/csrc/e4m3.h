// Numbers of 8 bits with a scale: code x 2^(scale - 127).
#pragma once
#include "device_utils.h"

namespace dcp {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// The scale's factor, as the conversions below take it: they look at its exponent alone.
__device__ __forceinline__ float scale_factor(uint32_t scale) { return __uint_as_float(min(max(scale, 1u), 254u) << 23); }

// Codes 2 HI, 2 HI + 1 of four as two bf16 numbers, exact: 4 significant bits, and 2^(scale - 127) moves the exponent.
template <bool HI> __device__ __forceinline__ uint32_t e4m3_to_bf16x2(uint32_t four, float factor) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, factor, HI));
}
template <bool HI> __device__ __forceinline__ f32x2_t e4m3_to_f32x2(uint32_t four) {
  return __builtin_bit_cast(f32x2_t, __builtin_amdgcn_cvt_pk_f32_fp8(four, HI));
}
// Four numbers as codes, rounded to nearest even; what is over 464, and NaN, becomes NaN.
__device__ __forceinline__ uint32_t f32x4_to_e4m3(float a, float b, float c, float d) {
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

// The sign bits of those of four codes that are not finite as bf16 and fp32 numbers: NaN, and with a scale s from 247 on what reaches 2^128 = 256 x 2^120, code 0x78,
// eight codes (a power of two) earlier for each further scale.
__device__ __forceinline__ uint32_t not_finite(uint32_t four, uint32_t scale) {
  const uint32_t least = scale < 247 ? 0x7f : 0x78 - 8 * (min(scale, 254u) - 247);
  return ((four & 0x7f7f7f7fu) + (0x80 - least) * 0x01010101u) & 0x80808080u;
}
__device__ __forceinline__ uint32_t without(uint32_t four, uint32_t signs) { return four & ~((signs >> 7) * 0xffu); }   // those as 0

// fp32 numbers go into products as three bf16 parts of 8 significant bits each: the upper half of the number, and of what is left.  What these give is what is left of part x of
// the number `of`; instead of nothing 2^-30 of the number, far below what fp32 sums hold, as an infinity that the parts multiply would become NaN with a part of 0.
__device__ __forceinline__ float upper(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
__device__ __forceinline__ float left_of_weight(float x, float of) { return fmaxf(x - upper(x), of * 0x1p-30f); }   // not negative
__device__ __forceinline__ float left_of_query(float x, float of) {                                                // may be infinite: all its parts are
  const float left = x - upper(x);
  return fabsf(of) == INFINITY ? of : left == 0.f ? of * 0x1p-30f : left;
}

// The least scale, from 10 on, whose 448 units reach a number with these bits (no sign, finite): 448 = 1.75 x 2^8.
__device__ __forceinline__ uint32_t least_scale(uint32_t bits) {
  const int32_t s = (int32_t)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u);
  return (uint32_t)max(s, 10);
}

}  // namespace dcp
