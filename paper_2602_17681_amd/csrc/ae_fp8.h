// ae_fp8.h — E4M3 codes with a binary32 scale for each block of 128: what the quantiser, the products that quantise on the
// way and the norms with 8-bit outputs share.
#pragma once

#include <float.h>

#include "ae_device.h"
#include "ae_rows.h"

namespace ae {

constexpr int BLK = 128;                 // elements that share a scale
constexpr float kCodeMax = 448.0f;       // largest magnitude of an E4M3 code
constexpr float kScaleMin = 1.17549435e-38f;

// Infinities are rare and cost the common case nothing: the maximum over all magnitudes (which passes NaN by) tells whether
// a block holds any.  If not, x * (1 / scale) is at most 448 (1 + 2^-23), which the conversion rounds to 448, and a NaN
// becomes the NaN code by itself; if so, the maximum is taken again over what is finite, and the products are cut off at 448.
__device__ __forceinline__ float finite_abs(float v) {
  const float a = fabsf(v);
  return a <= FLT_MAX ? a : 0.0f;
}
__device__ __forceinline__ float block_scale(float amax) { return fmaxf(amax / kCodeMax, kScaleMin); }
template <bool INF>
__device__ __forceinline__ float code_value(float v, float inv) {
  const float y = v * inv;
  if constexpr (!INF) return y;
  return y != y ? y : fminf(fmaxf(y, -kCodeMax), kCodeMax);
}
template <bool INF>
__device__ __forceinline__ float magnitude(float v) { return INF ? finite_abs(v) : fabsf(v); }
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

}  // namespace ae
