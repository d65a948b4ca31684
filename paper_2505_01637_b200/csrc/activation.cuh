// The activations of the linear layers and their slopes, in f32.
//   relu(z) = max(z, 0)                    gelu(z) = z Phi(z), Phi the normal distribution function
//   silu(z) = z / (1 + e^-z)               gelu_tanh(z) = z (1 + tanh u) / 2,
//                                          u = sqrt(2 / pi) (z + 0.044715 z^3)
// (1 + tanh u) / 2 = 1 / (1 + e^-2u), so gelu_tanh and silu share one form, z * p(t) with
// p(t) = 1 / (1 + e^-t).
// Phi by Hastings' approximation (Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26):
// erfc(x) = (a1 t + ... + a5 t^5) e^(-x^2), t = 1 / (1 + 0.3275911 x), x >= 0, absolute error below 1.5e-7,
// so Phi(-|z|) = erfc(|z| / sqrt 2) / 2 without cancellation.  It is free of branches: in an epilogue of
// 4096 x 4096 results the eight values a thread holds interleave, where erff (branches) left the epilogue
// longer than the products it follows (185 against 101 us without an activation).
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace morello {

enum { kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4, kActCount = 5 };

// 1 / x to within a unit or two in the last place; 0 for infinity.
__device__ __forceinline__ float fast_reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float fast_exp2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.402823466e38f;
// p(t) = 1 / (1 + e^-t), given t log2(e); the power may overflow to infinity, the quotient is then 0.
__device__ __forceinline__ float logistic2(float t_log2e) { return fast_reciprocal(1.f + fast_exp2(-t_log2e)); }

// The tail 1 - Phi(a) of the normal distribution, a >= 0 and moderate, and its bell e^(-a^2 / 2).
__device__ __forceinline__ float normal_tail(float a, float* bell) {
  const float t = fast_reciprocal(fmaf(0.23164189f, a, 1.f));        // 0.3275911 / sqrt 2
  float s = fmaf(t, 0.5307027145f, -0.7265760135f);                  // the coefficients halved
  s = fmaf(t, s, 0.7107068705f);
  s = fmaf(t, s, -0.142248368f);
  s = fmaf(t, s, 0.127414796f);
  *bell = fast_exp2(a * (-0.5f * kLog2e) * a);
  return s * t * *bell;
}

constexpr float kInvSqrt2Pi = 0.39894228040143268f;
constexpr float kTwoSqrt2OverPi = 1.5957691216057308f;   // 2 sqrt(2 / pi)
// Where |z| is past kTail every activation has reached its limits in f32.
constexpr float kTail = 100.f;

// Every result is free of branches and of inf * 0: at z = -inf the other factor is 0, so z is kept finite
// there (max with the lowest number; a NaN z, which max would swallow, is still in the other factor).
template <int kAct>
__device__ __forceinline__ float act_value(float z) {
  if constexpr (kAct == kActNone) return z;
  const float relu = z < 0.f ? 0.f : z;
  if constexpr (kAct == kActRelu) return relu;
  if constexpr (kAct == kActGelu) {
    // z Phi(z) = max(z, 0) - |z| (1 - Phi(|z|))
    float bell;
    const float a = fminf(fabsf(z), kTail);
    return fmaf(-a, normal_tail(a, &bell), relu);
  }
  if constexpr (kAct == kActGeluTanh)
    return fmaxf(z, kLowest) * logistic2(z * fmaf(0.044715f * kTwoSqrt2OverPi * kLog2e * z, z, kTwoSqrt2OverPi * kLog2e));
  return fmaxf(z, kLowest) * logistic2(z * kLog2e);
}
// act'(z), and act(z) beside it: both come from the same exponential.
template <int kAct>
__device__ __forceinline__ float act_slope(float z, float* value) {
  if constexpr (kAct == kActNone) {
    *value = z;
    return 1.f;
  }
  const float relu = z < 0.f ? 0.f : z;
  if constexpr (kAct == kActRelu) {
    *value = relu;
    return z > 0.f ? 1.f : (z != z ? z : 0.f);
  }
  float d;
  if constexpr (kAct == kActGelu) {
    float bell;
    const float a = fminf(fabsf(z), kTail);
    const float tail = normal_tail(a, &bell);
    *value = fmaf(-a, tail, relu);
    d = (z < 0.f ? tail : 1.f - tail) + copysignf(a, z) * kInvSqrt2Pi * bell;
    return z != z ? z : d;
  }
  // Past the tail p (1 - p) is 0; c is z held where its products stay finite.
  const float c = fminf(fmaxf(z, -kTail), kTail);
  if constexpr (kAct == kActGeluTanh) {
    const float p = logistic2(c * fmaf(0.044715f * kTwoSqrt2OverPi * kLog2e * c, c, kTwoSqrt2OverPi * kLog2e));
    *value = fmaxf(z, kLowest) * p;
    d = p + c * p * (1.f - p) * kTwoSqrt2OverPi * fmaf(3.f * 0.044715f * c, c, 1.f);
  } else {
    const float p = logistic2(c * kLog2e);
    *value = fmaxf(z, kLowest) * p;
    d = p * fmaf(c, 1.f - p, 1.f);
  }
  if (z != z) *value = z;
  return z != z ? z : d;
}

// f32 <-> bf16, the rounding of every 16-bit output: to nearest, ties to even.
__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ float bf16_value(uint16_t h) { return __uint_as_float((uint32_t)h << 16); }
__device__ __forceinline__ uint32_t bf16_pack(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint16_t bf16_round(float v) { return (uint16_t)bf16_pack(v, 0.f); }

}  // namespace morello
