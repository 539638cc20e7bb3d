// GELU(v) = v Phi(v) and its derivative by Phi(x) = 2^Q(x) for x = -|v| <= 0, Q of degree 11
// (tests/gelu_log_fit.py fits it): Phi within 2^-18 of itself for x >= -4, 2^-12 down to
// -12.9, x = -13 standing for all that is smaller. Two values at a time, 12 packed multiply-adds and
// an ex2 each; no cancellation, so small results are as exact as large ones. NaN stays NaN.
// (The 4-bit product holds the same constants beside its own packing.)
#pragma once

#include "tc_common.cuh"

namespace unif {
namespace gelu {

#define UNIF_K2(bits) ((uint64_t)(bits##u) << 32 | (uint64_t)(bits##u))
// x_i = -|v_i| (at least -13) and Phi(x_i).
__device__ __forceinline__ void phi_negative2(float v0, float v1, uint64_t& x, float& p0, float& p1) {
  float x0, x1;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(x0) : "f"(-fabsf(v0)), "f"(-13.f));
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(x1) : "f"(-fabsf(v1)), "f"(-13.f));
  x = tc::pk2(x0, x1);
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
  float q0, q1;
  tc::upk2(q, q0, q1);
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(p0) : "f"(q0));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(p1) : "f"(q1));
}
#undef UNIF_K2

// GELU of two values: max(v, 0) + x Phi(x).
__device__ __forceinline__ void gelu2(float& v0, float& v1) {
  uint64_t x;
  float p0, p1;
  phi_negative2(v0, v1, x, p0, p1);
  tc::upk2(tc::fma2(x, tc::pk2(p0, p1), tc::pk2(fmaxf(v0, 0.f), fmaxf(v1, 0.f))), v0, v1);
}

// Its derivative Phi(v) + v phi(v), phi(v) = e^(-v^2 / 2) / sqrt(2 pi): with x = -|v| and
// s = Phi(x) + x phi(x) it is s for v <= 0 and 1 - s for v > 0. Beyond 13 it is 0 or 1.
__device__ __forceinline__ void gelu_grad2(float v0, float v1, float& d0, float& d1) {
  uint64_t x;
  float p0, p1, x0, x1, e0, e1;
  phi_negative2(v0, v1, x, p0, p1);
  tc::upk2(x, x0, x1);
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(x0 * x0 * -0.72134752044448170f));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(x1 * x1 * -0.72134752044448170f));
  d0 = fmaf(x0 * 0.39894228040143268f, e0, p0);
  d1 = fmaf(x1 * 0.39894228040143268f, e1, p1);
  if (v0 > 0.f) d0 = 1.f - d0;
  if (v1 > 0.f) d1 = 1.f - d1;
}

}  // namespace gelu
}  // namespace unif
