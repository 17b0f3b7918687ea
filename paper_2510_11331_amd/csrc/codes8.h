// 8-bit numbers of the feed-forward network, on the device.
//
// Format: e4m3 codes (largest 448) with a power-of-two scale 2^(E - 127) per
// block of 128 entries of a row (activations) or of 128 x 128 entries
// (weights).  E is the smallest E >= 1 with amax <= 448 2^(E - 127), amax the
// largest magnitude of the block's finite entries; a code is v 2^(127 - E)
// rounded to nearest even (the product is exact, so there is one rounding),
// NaN and infinities become the NaN code.  A power of two costs nothing
// against amax / 448: a floating code's relative step is the same wherever its
// value lies, and the scaled matrix instruction takes the exponent byte as it is.
#pragma once

#include "sd_internal.h"

namespace sd {

// magnitude that counts for a block's maximum: 0 for NaN and infinities
__device__ __forceinline__ float finite_abs(float v) {
  const float a = fabsf(v);
  return a < INFINITY ? a : 0.f;
}

// E of a block with maximum amax = m 2^e (1 <= m < 2): 448 = 1.75 2^8, so E - 127
// is e - 8 for m <= 1.75, else e - 7: a carry out of the fraction field
__device__ __forceinline__ int block_exp(float amax) {
  return max((int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - 8, 1);
}
__device__ __forceinline__ float inv_scale(int E) { return __uint_as_float((uint32_t)(254 - E) << 23); }

// four codes (|v| inv <= 448 where finite; overflow, infinities and NaN give NaN)
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, lo, true);
}

// bf16 bits of f, rounded to nearest even (any f; v_cvt_pk_bf16_f32)
__device__ __forceinline__ uint32_t bf16_bits(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

}  // namespace sd
