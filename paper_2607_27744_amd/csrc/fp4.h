// Device side of the cache's 4-bit form (layer.h: Fp4Row): e2m1 values with a
// power-of-two scale (a byte of exponent) for 32 of them. The conversion
// instructions take the scale as the exponent of a float: 2^(E - 127) is the bits
// E << 23, E = 0 (a float of zero) is 2^-127, and E = 255 makes NaN of every value
// (checked on the card, as is that the rounding is to the nearest, ties to the even
// code, saturating at 6).
#pragma once

#include "common.h"
#include "layer.h"

namespace rocs {

__device__ __forceinline__ float fp4_scale(uint32_t e) { return __builtin_bit_cast(float, e << 23); }

// Eight values (a 32-bit word) as bf16, exactly.
__device__ __forceinline__ u32x4 fp4_to_bf16x8(uint32_t w, float scale) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
}

// Value j (0 .. 7) of a word, as a float.
__device__ __forceinline__ float fp4_value(uint32_t w, int j, float scale) {
  const uint32_t p = __builtin_bit_cast(
      uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w >> (4 * j), scale, 0));
  return bf16_lo(p);
}

// The scale byte of a block whose largest magnitude is m: the exponent that
// puts m in [4, 8), one more where m would pass 7 (nearer to 8 than to 6: kept
// at 6 it would be off by more than half the form's largest step). Kept within
// 1 .. 252: below, m is the smaller for it; above, values saturate at 6.
__device__ __forceinline__ uint32_t fp4_exponent(float m) {
  const uint32_t b = __builtin_bit_cast(uint32_t, m) & 0x7fffffffu;
  if (b >= 0x7f800000u) return 255u;
  const int e = (int)(b >> 23) - 2 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)min(max(e, 1), 252);
}

// Eight values to a word.
__device__ __forceinline__ uint32_t fp4_from_f32x8(const float (&x)[8], float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
  return w;
}

}  // namespace rocs
