// The activations of activation.cuh, two values an instruction where there is one for both (sums and products of pairs of
// f32; reciprocals, powers and comparisons are single).  The same formulas and roundings.
#pragma once

#include "activation.cuh"
#include "sm100.cuh"

namespace morello {

using sm100::f32x2;

// max(z, 0); NaN stays NaN.
__device__ __forceinline__ float relu_value(float z) {
  float r;
  asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(z));
  return r;
}
// 1 / (1 + 2^t)
__device__ __forceinline__ f32x2 logistic_pair(f32x2 t) {
  const float2 f = sm100::pair_values(t);
  const float2 d = sm100::pair_values(sm100::add2(sm100::pair_of(fast_exp2(f.x), fast_exp2(f.y)), sm100::pair_of(1.f)));
  return sm100::pair_of(fast_reciprocal(d.x), fast_reciprocal(d.y));
}

template <int kAct>
__device__ __forceinline__ f32x2 act_pair(f32x2 z) {
  using namespace sm100;
  if constexpr (kAct == kActNone) return z;
  const float2 f = pair_values(z);
  if constexpr (kAct == kActRelu || kAct == kActGelu) {
    const f32x2 relu = pair_of(relu_value(f.x), relu_value(f.y));
    if constexpr (kAct == kActRelu) return relu;
    // max(z, 0) - |z| (1 - Phi(|z|)), the tail as normal_tail() has it
    const f32x2 a = pair_of(fminf(fabsf(f.x), kTail), fminf(fabsf(f.y), kTail));
    const float2 q = pair_values(fma2(a, pair_of(0.23164189f), pair_of(1.f)));
    const f32x2 t = pair_of(fast_reciprocal(q.x), fast_reciprocal(q.y));
    f32x2 s = fma2(t, pair_of(0.5307027145f), pair_of(-0.7265760135f));
    s = fma2(t, s, pair_of(0.7107068705f));
    s = fma2(t, s, pair_of(-0.142248368f));
    s = fma2(t, s, pair_of(0.127414796f));
    const float2 e = pair_values(mul2(mul2(a, pair_of(-0.5f * kLog2e)), a));
    const f32x2 tail = mul2(mul2(s, t), pair_of(fast_exp2(e.x), fast_exp2(e.y)));
    return fma2(mul2(a, pair_of(-1.f)), tail, relu);
  }
  const f32x2 kept = pair_of(fmaxf(f.x, kLowest), fmaxf(f.y, kLowest));
  if constexpr (kAct == kActGeluTanh) {
    const f32x2 u = fma2(mul2(z, pair_of(-0.044715f * kTwoSqrt2OverPi * kLog2e)), z, pair_of(-kTwoSqrt2OverPi * kLog2e));
    return mul2(kept, logistic_pair(mul2(z, u)));
  }
  return mul2(kept, logistic_pair(mul2(z, pair_of(-kLog2e))));
}
template <int kAct, int kCount>
__device__ __forceinline__ void act_pairs(f32x2 (&v)[kCount]) {
#pragma unroll
  for (int i = 0; i < kCount; ++i) v[i] = act_pair<kAct>(v[i]);
}
template <int kCount>
__device__ __forceinline__ void act_pairs_by(int act, f32x2 (&v)[kCount]) {
  if (act == kActNone) return;
  if (act == kActRelu) act_pairs<kActRelu>(v);
  else if (act == kActGelu) act_pairs<kActGelu>(v);
  else if (act == kActGeluTanh) act_pairs<kActGeluTanh>(v);
  else act_pairs<kActSilu>(v);
}

}  // namespace morello
