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

// 2^-e of a scale byte (1..247 by construction: a normal number).
__device__ __forceinline__ float fp8_inverse(uint32_t byte) {
  return __builtin_bit_cast(float, (254u - byte) << 23);
}

// Four values, times inv, as e4m3 bytes (the first in the lowest). An infinity
// is turned into NaN first: what the conversion makes of it is a mode's choice.
__device__ __forceinline__ uint32_t fp8_pack4(float a, float b, float c, float d, float inv) {
  auto one = [inv](float x) {
    x *= inv;
    return __builtin_fabsf(x) <= 448.0f ? x : __builtin_nanf("");
  };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(one(a), one(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(one(c), one(d), w, true);
}

// Largest of v over each row of 16 lanes, in all of them.
__device__ __forceinline__ float row16_max(float v) {
  v = fmaxf(v, dpp<kDppXor8>(v));
  v = fmaxf(v, dpp<kDppMirror8>(v));
  v = fmaxf(v, dpp<kDppXor2>(v));
  return fmaxf(v, dpp<kDppXor1>(v));
}

}  // namespace f3c
