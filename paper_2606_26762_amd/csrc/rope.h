// Rotary positions: the rotation that the readout (query.hip) and protokv_rotate
// (tokens.hip) share.
#pragma once

#include <hip/hip_runtime.h>

namespace pkv {

// cos and sin of the rotary angle pos * inv (inv = theta^(-2i/D)): the angle
// in float64, whole turns taken off in float64, the rest (|r| <= pi) to
// float32 sincos.  Stream positions reach 10^6 and more, where a float32
// angle would already be off by tenths of a radian.
__device__ __forceinline__ void rope_cs(double pos, double inv, float& c, float& s) {
  const double a = pos * inv;
  const double turns = rint(a * 0.15915494309189535);  // 1 / (2 pi)
  const float r = (float)fma(-turns, 6.283185307179586, a);
  sincosf(r, &s, &c);
}

// Rotate-half rotation of the pair (x1 = dim i, x2 = dim i + D/2):
// lo = x1 c - x2 s, hi = x2 c + x1 s (float32, one rounding per operation).
__device__ __forceinline__ void rope_pair(float x1, float x2, float c, float s, float& lo, float& hi) {
  lo = x1 * c - x2 * s;
  hi = x2 * c + x1 * s;
}

}  // namespace pkv
