// Heads in 8 bits: E4M3 codes with a power of two for each head of a token.
#pragma once

#include <type_traits>

#include "thrift_device.h"

namespace thrift {

// x if it is finite, otherwise 0
__device__ __forceinline__ float finite_or_zero(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? 0.f : x; }

// e of the scale 2^e of a head whose largest finite magnitude is a: the least with a <= 448 * 2^e = 1.75 * 2^(e + 8), read off a's bits.  The
// upper end, 120, is that of fp32's largest number.  The lower one keeps products of a probability and the scale normal numbers down to
// probabilities of 2^-26; heads that it holds up are below 2^-91 in all elements.
__device__ __forceinline__ int e4m3_exponent(float a) {
  const uint32_t bits = __float_as_uint(a);
  const int e = (int)(bits >> 23) - 135 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return bits == 0 ? 0 : max(e, -100);
}

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// What a scale byte stands for; 0, which no head has, becomes 0
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Two elements times `inv` = 2^-e as codes in the half SEL of old, rounded to nearest even (one product with a power of two in front, exact but
// below 2^-126).  What has no code, NaN and infinities, becomes NaN in the conversion.
template <bool SEL>
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t old, float x, float y, float inv) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x * inv, y * inv, (int)old, SEL);
}

// The scale in byte i of a register
__device__ __forceinline__ float scale_in(uint32_t bytes, int i) {
  return __uint_as_float((i == 0 ? bytes << 23 : i == 1 ? bytes << 15 : i == 2 ? bytes << 7 : bytes >> 1) & 0x7f800000u);
}

// Codes 2 SEL and 2 SEL + 1 of a register as 16-bit numbers, exactly
template <typename T, bool SEL>
__device__ __forceinline__ uint32_t widen8(uint32_t codes) {
  if constexpr (std::is_same_v<T, F16>) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, 1.f, SEL));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, SEL));
}

// Eight codes times a scale as 16-bit numbers
template <typename T>
__device__ __forceinline__ v4i widen_chunk(v2i codes, float scale) {
  v4i y;
#pragma unroll
  for (int d = 0; d < 2; ++d) {
    if constexpr (std::is_same_v<T, F16>) {
      y[2 * d] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((uint32_t)codes[d], scale, false));
      y[2 * d + 1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((uint32_t)codes[d], scale, true));
    } else {
      y[2 * d] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[d], scale, false));
      y[2 * d + 1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[d], scale, true));
    }
  }
  return y;
}

// Codes 2 SEL and 2 SEL + 1 of a register, times a scale
template <bool SEL>
__device__ __forceinline__ float2 e4m3_values(uint32_t codes, float scale) {
  const auto x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, 1.f, SEL);
  return make_float2(x[0] * scale, x[1] * scale);
}

}  // namespace thrift
