// Codes and scales of the paged cache's blocks of 64 tokens and head.
#pragma once

#include "mw_device.h"

namespace mw {

// The scale of a block: 2^e with the least e such that amax <= 448 * 2^e, clamped to [-100, 100].
// A power of two makes the division by it, the product with it and a later change of it exact
// (up to e4m3's subnormals), and costs e4m3, which is a floating-point format, no precision.
__device__ __forceinline__ int block_exponent(float amax) {
  const unsigned u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);  // 448 = 1.75 * 2^8
  return min(max(e, -100), 100);
}
__device__ __forceinline__ float pow2(int e) { return e < -126 ? 0.f : __uint_as_float((unsigned)(e + 127) << 23); }

// +-448 at most; NaN stays NaN.
__device__ __forceinline__ float clamp448(float x) { return x == x ? fminf(fmaxf(x, -448.f), 448.f) : x; }

// Eight values -> codes, and back.
__device__ __forceinline__ u32x2 encode8(const float* x, float mul) {
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = clamp448(x[j] * mul);
  u32x2 r;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w], y[4 * w + 1], 0, false);
    r[w] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w + 2], y[4 * w + 3], lo, true);
  }
  return r;
}

__device__ __forceinline__ void decode8(const u32x2& u, float* x) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)u[j], false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)u[j], true);
    x[4 * j] = lo[0];
    x[4 * j + 1] = lo[1];
    x[4 * j + 2] = hi[0];
    x[4 * j + 3] = hi[1];
  }
}

}  // namespace mw
