// Codes and scales of 8-bit activation checkpoints (act8.hip says what they are), for the kernels
// that write them.
#pragma once

#include <math.h>

#include "common.h"

namespace merak {

constexpr int kScaleBlock = 32;
constexpr int kMinScale = 127 - 117;  // smallest scale byte
constexpr float kLargest = 0x1.ep127f;  // 240 * 2^120

// Scale byte for a block whose largest finite |x| has the bits `m`: exponent - 8,
// plus one where the significand is above 1.75 = 448 / 256.
__device__ __forceinline__ int scale_byte(uint32_t m) {
  const int b = (int)(m >> 23) - 8 + ((m & 0x7fffffu) > 0x600000u);
  return max(b, kMinScale);
}

// Bits of |x| for the block's maximum: 0 for NaN and infinities.
__device__ __forceinline__ uint32_t finite_mag(float x) {
  const uint32_t m = __float_as_uint(x) & 0x7fffffffu;
  return m < 0x7f800000u ? m : 0u;
}

// Four codes; inv = 1 / scale.
__device__ __forceinline__ uint32_t encode4(const float v[4], float inv) {
  float s[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float c = fminf(fmaxf(v[e], -kLargest), kLargest);
    s[e] = finite_mag(v[e]) == (__float_as_uint(v[e]) & 0x7fffffffu) ? c * inv : NAN;
  }
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(s[0], s[1], 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(s[2], s[3], r, true);
  return (uint32_t)r;
}

}  // namespace merak
