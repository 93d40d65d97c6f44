// 8-bit rows: OCP e4m3 values with one power-of-two scale (E8M0 byte, 2^(byte -
// 127)) per block of 128 along the row.
//
// A block's scale is the smallest 2^e, e in [-126, 127], with |x| <= 448 * 2^e
// for every finite x of the block, so nothing saturates, and x * 2^-e is exact:
// the rounding to e4m3 (nearest even, half a step: 2^-4 relative) is the only
// one. The matrix cores take the scale byte as an operand. NaN and infinities
// do not count towards the scale and become e4m3's NaN.
#pragma once

#include "common.h"

namespace f3c {

constexpr int kFp8Block = 128;

typedef int i32x8 __attribute__((ext_vector_type(8)));

// |x| where it is finite, else 0.
__device__ __forceinline__ float finite_abs(float x) {
  const float a = __builtin_fabsf(x);
  return a < __builtin_inff() ? a : 0.0f;
}

// Scale byte of a block whose largest finite magnitude is amax. 448 = 1.75 *
// 2^8: a mantissa above 1.75 carries into the exponent field.
__device__ __forceinline__ uint32_t fp8_scale_byte(float amax) {
  const int e = (int)((__builtin_bit_cast(uint32_t, amax) + 0x1fffffu) >> 23) - 8;
  return (uint32_t)(e < 1 ? 1 : e);
}

// 2^e of a scale byte (1..247 by construction: a normal number).
__device__ __forceinline__ float fp8_scale(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// Four finite values or NaNs over 2^e (the scale as a float) as e4m3 bytes, the
// first in the lowest: the conversion divides by the scale, exactly, and rounds
// once, to nearest even; nothing is out of range of a scale of fp8_scale_byte.
typedef short s16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t fp8_pack4(float a, float b, float c, float d, float scale) {
  s16x2 w{0, 0};
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, scale, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, w);
}

// x, an infinity as NaN (what the conversion makes of it is a mode's choice).
__device__ __forceinline__ float fp8_no_inf(float x) {
  return __builtin_fabsf(x) < __builtin_inff() ? x : __builtin_nanf("");
}

// Largest of v over each row of 16 lanes, in all of them.
__device__ __forceinline__ float row16_max(float v) {
  v = fmaxf(v, dpp<kDppXor8>(v));
  v = fmaxf(v, dpp<kDppMirror8>(v));
  v = fmaxf(v, dpp<kDppXor2>(v));
  return fmaxf(v, dpp<kDppXor1>(v));
}

}  // namespace f3c
