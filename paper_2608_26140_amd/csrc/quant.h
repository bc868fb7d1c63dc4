// The 8-bit KV cache's number format: e4m3 codes and one power-of-two scale
// for every block of consecutive slots and KV head.
//
// The smallest exponent e with amax <= 448 * 2^e needs no logarithm: 448 is
// 1.75 * 2^8, so e is amax's own exponent less 8, one more where its
// significand exceeds 1.75, which adding the rest of the significand's range
// (0x1FFFFF) carries into the exponent field.  e stays within [-117, 119], so
// that every code times its scale, the smallest subnormal (2^-9) and the
// largest value (1.75 * 2^8) included, is a bf16 number that is neither
// subnormal nor infinite; larger values saturate.
#pragma once

#include "device.h"

namespace acache {

constexpr float kMaxCode = 448.f;
constexpr int kMinScaleByte = 127 - 117, kMaxScaleByte = 127 + 119;

// The scale's exponent field (e + 127) for the largest finite magnitude.
__device__ __forceinline__ int scale_byte(float amax) {
  const int b = (int)((__float_as_uint(amax) + 0x1FFFFFu) >> 23) - 8;
  return min(max(b, kMinScaleByte), kMaxScaleByte);
}
__device__ __forceinline__ float pow2_byte(int b) { return __uint_as_float((uint32_t)b << 23); }
// A scale as it is read: the power of two at or below it.
__device__ __forceinline__ float pow2_below(float scale) {
  return __uint_as_float(__float_as_uint(scale) & 0xFF800000u);
}

// Four codes of x * inv, rounded to nearest even; an infinity or a NaN gives
// NaN (e4m3 has no infinity).
__device__ __forceinline__ float code_arg(float x, float inv) {
  const float y = fminf(fmaxf(x * inv, -kMaxCode), kMaxCode);
  return fabsf(x) < INFINITY ? y : __uint_as_float(0x7FC00000u);
}
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ void decode4(uint32_t w, float (&v)[4]) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  v[0] = lo[0];
  v[1] = lo[1];
  v[2] = hi[0];
  v[3] = hi[1];
}

}  // namespace acache
