// Rows in 8-bit floating point (E4M3) under a scale each: the scale of a row and the codes of
// its values. The scale is 2^e with the smallest e (at least -126) for which no value of
// the row is above 448 2^e, so that scaling is exact, nothing saturates, and codes are the same
// on every machine. (A scale of max / 448 would round twice and use the range a factor of two
// better at most, which a floating-point code does not gain from but at its small end.)
#pragma once

#include <stdint.h>

namespace unif {
namespace fp8 {

// From the bits of the row's largest absolute value: the scale's bits, and what its values
// are multiplied by (0 for rows with an infinity or NaN, whose scale is NaN and codes 0).
__device__ __forceinline__ float row_scale(uint32_t most, float& by) {
  const int exponent = (int)(most >> 23);
  if (exponent == 255) {
    by = 0.f;
    return __uint_as_float(0x7fffffffu);
  }
  const int s = max(exponent - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0), 1);  // 448 = 1.75 2^8
  by = __uint_as_float((uint32_t)(254 - s) << 23);
  return __uint_as_float((uint32_t)s << 23);
}

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Two values to codes, the first in the low byte (rounded to nearest even).
__device__ __forceinline__ uint32_t codes2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// Eight scaled values to codes; those of a row without finite scale are 0.
__device__ __forceinline__ uint2 codes8(const float (&v)[8], float by) {
  if (by == 0.f) return make_uint2(0u, 0u);
  return make_uint2(codes2(v[0] * by, v[1] * by) | codes2(v[2] * by, v[3] * by) << 16,
                    codes2(v[4] * by, v[5] * by) | codes2(v[6] * by, v[7] * by) << 16);
}

}  // namespace fp8
}  // namespace unif
