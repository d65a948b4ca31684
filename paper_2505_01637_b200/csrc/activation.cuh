// The activations of the linear layers and their slopes, in f32.
//   relu(z) = max(z, 0)                    gelu(z) = z Phi(z), Phi(z) = (1 + erf(z / sqrt 2)) / 2
//   silu(z) = z / (1 + e^-z)               gelu_tanh(z) = z (1 + tanh u) / 2,
//                                          u = sqrt(2 / pi) (z + 0.044715 z^3)
// (1 + tanh u) / 2 = 1 / (1 + e^-2u), so gelu_tanh and silu share one form, z * p(t) with
// p(t) = 1 / (1 + e^-t).
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace morello {

enum { kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4, kActCount = 5 };

// p(t) = 1 / (1 + e^-t); e^-t may overflow to infinity, the quotient is then 0.
__device__ __forceinline__ float logistic(float t) { return __fdividef(1.f, 1.f + __expf(-t)); }

constexpr float kSqrtHalf = 0.70710678118654752f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;
constexpr float kTwoSqrt2OverPi = 1.5957691216057308f;   // 2 sqrt(2 / pi)

// Beyond kTail every one of them has reached its limits in f32 (z or 0, slope 1 or 0): the limits are
// returned there, so that an infinite z gives them too instead of inf * 0.  NaN stays NaN.
constexpr float kTail = 100.f;

template <int kAct>
__device__ __forceinline__ float act_value(float z) {
  if constexpr (kAct == kActNone) return z;
  if constexpr (kAct == kActRelu) return z < 0.f ? 0.f : z;
  if (z < -kTail) return 0.f;
  if constexpr (kAct == kActGelu) return 0.5f * z * (1.f + erff(z * kSqrtHalf));
  if constexpr (kAct == kActGeluTanh)
    return z > kTail ? z : z * logistic(kTwoSqrt2OverPi * (z + 0.044715f * z * z * z));
  return z * logistic(z);
}
template <int kAct>
__device__ __forceinline__ float act_slope(float z) {
  if constexpr (kAct == kActNone) return 1.f;
  if constexpr (kAct == kActRelu) return z > 0.f ? 1.f : (z != z ? z : 0.f);
  if (fabsf(z) > kTail) return z > 0.f ? 1.f : 0.f;
  if constexpr (kAct == kActGelu)
    return 0.5f * (1.f + erff(z * kSqrtHalf)) + z * kInvSqrt2Pi * __expf(-0.5f * z * z);
  if constexpr (kAct == kActGeluTanh) {
    const float p = logistic(kTwoSqrt2OverPi * (z + 0.044715f * z * z * z));
    return p + z * p * (1.f - p) * kTwoSqrt2OverPi * (1.f + 3.f * 0.044715f * z * z);
  }
  const float p = logistic(z);
  return p * (1.f + z * (1.f - p));
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
