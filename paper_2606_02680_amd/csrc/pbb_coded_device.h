// Device-side helpers of the 8-bit paged cache: rows of e4m3 codes with one power of two each.
//
// A row's scale byte b stands for 2^(b - 127); its values are code times that.  The rows that an append
// writes have the least power 2^e (e from kScaleLo to kScaleHi) under which the row's largest finite
// magnitude is at most 448, the largest code's: so codes use the whole range, and scaling rounds nothing.
#pragma once

#include "pbb_device.h"

namespace pbb {

constexpr int kScaleLo = -100, kScaleHi = 119;   // (2^119 * 448 is above half the largest bf16 value)
constexpr float kCodeMost = 448.0f;

// The exponent for a row whose largest finite magnitude has these bits, at most `hi`.
__device__ __forceinline__ int scale_exponent(uint32_t most, int hi) {
  // 448 = 1.75 * 2^8: one more where the significand is above 1.75
  const int e = (int)(most >> 23) - 135 + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(max(e, kScaleLo), hi);
}
// 2^e for e of kScaleLo .. kScaleHi, their negatives, or a scale byte less 127.
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// The bits of a value's magnitude where it is finite, 0 where it is not.
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t m = __float_as_uint(x) & 0x7FFFFFFFu;
  return m < 0x7F800000u ? m : 0u;
}

// Codes of four values (already divided by the row's power of two, none finite above 448), nearest, ties
// to even; infinities and NaN become NaN.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// A finite value cut to the largest code's.
__device__ __forceinline__ float cut_finite(float x) {
  const float y = __builtin_amdgcn_fmed3f(x, -kCodeMost, kCodeMost);
  return finite_bits(x) != 0u ? y : x;
}

// Two codes (the low or the high half of w) times scale, a power of two: exact in bf16, one instruction.
template <bool HIGH>
__device__ __forceinline__ uint32_t values2(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HIGH));
}

}  // namespace pbb
