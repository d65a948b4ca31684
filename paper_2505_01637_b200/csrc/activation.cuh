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
// p(t) = 1 / (1 + e^-t); e^-t may overflow to infinity, the quotient is then 0.
__device__ __forceinline__ float logistic(float t) { return fast_reciprocal(1.f + __expf(-t)); }

constexpr float kSqrtHalf = 0.70710678118654752f;
// Phi(z), and e^(-z^2 / 2) for the slope.
__device__ __forceinline__ float normal_cdf(float z, float* bell) {
  const float x = fabsf(z) * kSqrtHalf;
  const float t = fast_reciprocal(fmaf(0.3275911f, x, 1.f));
  float s = fmaf(t, 1.061405429f, -1.453152027f);
  s = fmaf(t, s, 1.421413741f);
  s = fmaf(t, s, -0.284496736f);
  s = fmaf(t, s, 0.254829592f);
  *bell = __expf(-x * x);
  const float tail = 0.5f * s * t * *bell;
  return z < 0.f ? tail : 1.f - tail;
}

constexpr float kInvSqrt2Pi = 0.39894228040143268f;
constexpr float kTwoSqrt2OverPi = 1.5957691216057308f;   // 2 sqrt(2 / pi)

// Beyond kTail every one of them has reached its limits in f32 (z or 0, slope 1 or 0): the limits are
// returned there, so that an infinite z gives them too instead of inf * 0.  NaN stays NaN.
constexpr float kTail = 100.f;

template <int kAct>
__device__ __forceinline__ float act_value(float z) {
  if constexpr (kAct == kActNone) return z;
  if constexpr (kAct == kActRelu) return z < 0.f ? 0.f : z;
  float p;
  if constexpr (kAct == kActGelu) {
    float bell;
    p = normal_cdf(z, &bell);
  } else if constexpr (kAct == kActGeluTanh) {
    p = logistic(kTwoSqrt2OverPi * fmaf(0.044715f * z * z, z, z));
  } else {
    p = logistic(z);
  }
  return z < -kTail ? 0.f : z > kTail ? z : z * p;
}
template <int kAct>
__device__ __forceinline__ float act_slope(float z) {
  if constexpr (kAct == kActNone) return 1.f;
  if constexpr (kAct == kActRelu) return z > 0.f ? 1.f : (z != z ? z : 0.f);
  float d;
  if constexpr (kAct == kActGelu) {
    float bell;
    const float phi = normal_cdf(z, &bell);
    d = phi + z * kInvSqrt2Pi * bell;
  } else if constexpr (kAct == kActGeluTanh) {
    const float p = logistic(kTwoSqrt2OverPi * fmaf(0.044715f * z * z, z, z));
    d = p + z * p * (1.f - p) * kTwoSqrt2OverPi * (1.f + 3.f * 0.044715f * z * z);
  } else {
    const float p = logistic(z);
    d = p * (1.f + z * (1.f - p));
  }
  return z < -kTail ? 0.f : z > kTail ? 1.f : d;
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
