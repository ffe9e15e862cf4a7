// OCP e4m3 codes with power-of-two block scales: the number format of the
// 8-bit cache (gfx950 only).
//
// A scale 2^e is stored as the byte e + 127, which is also the exponent field
// of the fp32 number 2^e. A code has four significant bits, so code * 2^e is
// exact in bf16 (and fp32): the conversion to the matrix operands rounds
// nothing.
#pragma once

#include "hsa_device.h"
#include "hsa_kernels.h"

namespace hsa {

constexpr int kScaleTok = HSA_CACHE8_BLOCK;  // tokens of a page that share a scale
// Exponents of a scale: 448 * 2^120 is the largest a finite fp32 number needs; from
// 2^-100 on, codes times the scale stay normal numbers.
constexpr int kScaleMin = -100, kScaleMax = 120;
constexpr float kCodeMax = 448.f;  // largest e4m3 number

typedef uint32_t u32x4a8 __attribute__((ext_vector_type(4), aligned(8)));
typedef uint32_t u32x2a8 __attribute__((ext_vector_type(2), aligned(8)));

// 2^e of a stored exponent byte. Every byte gives a finite number, so that the zero codes
// in the place of tokens past a sequence's end stay zeros whatever its memory holds.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(min(max(byte, 1u), 254u) << 23); }
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(clampi(e, -126, 127) + 127) << 23); }

// Eight codes (low byte first) times a power of two, as a bf16 matrix operand.
__device__ __forceinline__ u32x4 codes_to_bf16(uint32_t lo, uint32_t hi, float scale) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, scale, false);
  const auto b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, scale, true);
  const auto c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, scale, false);
  const auto d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, scale, true);
  return u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
               __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)};
}

// Codes of numbers in units of a scale 2^e, rounded to nearest even; low byte first. The
// caller's scale leaves no finite number above the largest code; saturate()
// takes the infinities there first (e4m3 has none). NaN gives a NaN code.
__device__ __forceinline__ float saturate(float x, float most) { return x != x ? x : fminf(fmaxf(x, -most), most); }
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t codes2(float a, float b, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(i16x2{0, 0}, a, b, scale, false));
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float scale) {
  i16x2 w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(i16x2{0, 0}, a, b, scale, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, w);
}
// the same of two pairs of bf16 numbers
__device__ __forceinline__ uint32_t codes4_bf16(uint32_t ab, uint32_t cd, float scale) {
  i16x2 w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(i16x2{0, 0}, __builtin_bit_cast(bf16x2, ab), scale, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, cd), scale, true);
  return __builtin_bit_cast(uint32_t, w);
}
// One code as a number.
__device__ __forceinline__ float code_to_f32(uint32_t byte) { return __builtin_amdgcn_cvt_f32_fp8((int)byte, 0); }

// Smallest exponent e with amax <= 448 * 2^e, within the range of a scale. 448 =
// 1.75 * 2^8: amax = m * 2^k with m in [1, 2) needs k - 8, or k - 7 if m > 1.75.
// amax = 0 (or subnormal) gives the smallest.
__device__ __forceinline__ int scale_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int k = (int)(u >> 23) - 127;
  return clampi(k - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0), kScaleMin, kScaleMax);
}

}  // namespace hsa
