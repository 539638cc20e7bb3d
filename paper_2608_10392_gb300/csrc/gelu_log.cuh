// GELU(v) = v Phi(v) and its derivative by Phi(x) = 2^Q(x) for x = -|v| <= 0 (x = -13 stands for all
// that is smaller): no cancellation, so small results are as exact as large ones. NaN stays NaN.
// Two values at a time in packed multiply-adds. Fits: tests/gelu_log_fit.py (its algorithm; the
// degrees and weights are below).
#pragma once

#include "tc_common.cuh"

namespace unif {
namespace gelu {

#define UNIF_K2(bits) ((uint64_t)(bits##u) << 32 | (uint64_t)(bits##u))
// x_i = -|v_i|, at least -13.
__device__ __forceinline__ uint64_t negative2(float v0, float v1) {
  float x0, x1;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(x0) : "f"(-fabsf(v0)), "f"(-13.f));
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(x1) : "f"(-fabsf(v1)), "f"(-13.f));
  return tc::pk2(x0, x1);
}
__device__ __forceinline__ void two_to(uint64_t q, float& p0, float& p1) {
  float q0, q1;
  tc::upk2(q, q0, q1);
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(p0) : "f"(q0));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(p1) : "f"(q1));
}

// GELU of two values, max(v, 0) + x Phi(x), for results that are rounded to bf16: Q of degree 8, its
// error the same everywhere, leaves Phi within 2^-12.8 of itself, a twenty-eighth of the result's rounding by 2^-8.
// (A product's storing warps run this chain between the load and the store of a piece: 65,536 x 1,024 to 4,096 in 8
// bits takes 250 us, with degree 11 275, without GELU 190; 12,608 x 384 to 1,536 in bf16 22.8, 24.2 and 17.3.)
__device__ __forceinline__ void gelu2(float& v0, float& v1) {
  const uint64_t x = negative2(v0, v1);
  uint64_t q = UNIF_K2(0x32ed9bf9);         // g8
  q = tc::fma2(q, x, UNIF_K2(0x35eb8204));  // g7
  q = tc::fma2(q, x, UNIF_K2(0x38495417));  // g6
  q = tc::fma2(q, x, UNIF_K2(0x3a441950));  // g5
  q = tc::fma2(q, x, UNIF_K2(0x3bf3df33));  // g4
  q = tc::fma2(q, x, UNIF_K2(0x3d5064c2));  // g3
  q = tc::fma2(q, x, UNIF_K2(0xbeece188));  // g2
  q = tc::fma2(q, x, UNIF_K2(0x3f931688));  // g1
  q = tc::fma2(q, x, UNIF_K2(0xbf80057d));  // g0
  float p0, p1;
  two_to(q, p0, p1);
  tc::upk2(tc::fma2(x, tc::pk2(p0, p1), tc::pk2(fmaxf(v0, 0.f), fmaxf(v1, 0.f))), v0, v1);
}

// Its derivative Phi(v) + v phi(v), phi(v) = e^(-v^2 / 2) / sqrt(2 pi): with x = -|v| and
// s = Phi(x) + x phi(x) it is s for v <= 0 and 1 - s for v > 0. Beyond 13 it is 0 or 1.
// Q of degree 11, Phi within 2^-18 of itself for x >= -4 and 2^-12 beyond (the 4-bit product holds the
// same polynomial): sums over tokens are taken of it in fp32.
__device__ __forceinline__ void gelu_grad2(float v0, float v1, float& d0, float& d1) {
  const uint64_t x = negative2(v0, v1);
  uint64_t q = UNIF_K2(0xae8f0e53);         // q11
  q = tc::fma2(q, x, UNIF_K2(0xb191c94c));  // q10
  q = tc::fma2(q, x, UNIF_K2(0xb3f84d3a));  // q9
  q = tc::fma2(q, x, UNIF_K2(0xb5def6f2));  // q8
  q = tc::fma2(q, x, UNIF_K2(0xb74c0539));  // q7
  q = tc::fma2(q, x, UNIF_K2(0xb738e2e6));  // q6
  q = tc::fma2(q, x, UNIF_K2(0x3a367766));  // q5
  q = tc::fma2(q, x, UNIF_K2(0x3c03d9e8));  // q4
  q = tc::fma2(q, x, UNIF_K2(0x3d5ae7de));  // q3
  q = tc::fma2(q, x, UNIF_K2(0xbeeae20c));  // q2
  q = tc::fma2(q, x, UNIF_K2(0x3f935a21));  // q1
  q = tc::fma2(q, x, UNIF_K2(0xbf7fffd6));  // q0
  float p0, p1, x0, x1, e0, e1;
  two_to(q, p0, p1);
  tc::upk2(x, x0, x1);
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(x0 * x0 * -0.72134752044448170f));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(x1 * x1 * -0.72134752044448170f));
  d0 = fmaf(x0 * 0.39894228040143268f, e0, p0);
  d1 = fmaf(x1 * 0.39894228040143268f, e1, p1);
  if (v0 > 0.f) d0 = 1.f - d0;
  if (v1 > 0.f) d1 = 1.f - d1;
}

#undef UNIF_K2

}  // namespace gelu
}  // namespace unif
