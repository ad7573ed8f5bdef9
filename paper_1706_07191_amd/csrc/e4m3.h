// Numbers of 8 bits (e4m3: four bits of exponent, three of fraction, largest 448, no infinities) with a power-of-two scale for each block.
#pragma once
#include "common.h"

namespace brsvd {

constexpr int kBlock = 128;      // numbers of a row that share a scale

// The least e >= -126 with top <= 448 * 2^e, 0 for top = 0; top >= 0 is finite.  448 = 1.75 * 2^8, so it is read off the bits.  A power of two as the
// scale costs e4m3 nothing but a binade at its lower end, and dividing by it rounds nothing: a number is rounded once.
__device__ __forceinline__ int block_exponent(float top) {
  const uint32_t b = __float_as_uint(top);
  const int e = (int)(b >> 23) - 135 + ((b & 0x7fffffu) > 0x600000u);
  return top > 0.f ? (e < -126 ? -126 : e) : 0;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// |x| for the largest of a block: what is not finite does not count
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a <= 3.402823466e38f ? a : 0.f;
}
// Four numbers, scaled, to the nearest e4m3 (ties to even; NaN for what is not finite).
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  return (uint32_t)r;
}

}  // namespace brsvd
