// Activations of the FFN operators and their derivatives, in fp32.
//
//   relu(z) = max(z, 0)              silu(z) = z s(z), s the logistic function
//   gelu(z) = z s(2u), u = sqrt(2/pi) (z + 0.044715 z^3)   (the tanh form:
//             (1 + tanh u) / 2 = s(2u))
//
// s(x) = 1 / (1 + 2^(-x log2 e)) is one v_exp_f32 and one v_rcp_f32 (1 ulp
// each), so an activation is within a few ulp of fp32 wherever it is not
// tiny; a large negative x gives 1 / inf = 0. NaN stays NaN.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "../host/plan.hpp"

namespace ccl {

__device__ __forceinline__ float logistic(float x) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504089f * x));
}

constexpr float kGelu2 = 1.59576912161f;   // 2 sqrt(2/pi)

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if constexpr (ACT == ACT_RELU) return z < 0.f ? 0.f : z;
  if constexpr (ACT == ACT_GELU) return z * logistic(kGelu2 * z * (1.f + 0.044715f * z * z));
  if constexpr (ACT == ACT_SILU) return z * logistic(z);
  return z;
}

// Value and derivative. The derivative is formed at z clamped to +-100, where
// both functions are 0 or z to the last bit: beyond, its factors would meet as
// 0 * inf. With s = s(v): s' = s (1 - s) v'.
template <int ACT>
__device__ __forceinline__ float act_value_grad(float z, float* grad) {
  if constexpr (ACT == ACT_RELU) {
    *grad = z < 0.f ? 0.f : (z > 0.f ? 1.f : z);   // 0 at 0, NaN at NaN
    return z < 0.f ? 0.f : z;
  }
  if constexpr (ACT == ACT_GELU || ACT == ACT_SILU) {
    const float c = z > 100.f ? 100.f : (z < -100.f ? -100.f : z);
    const float v = ACT == ACT_SILU ? c : kGelu2 * c * (1.f + 0.044715f * c * c);
    const float dv = ACT == ACT_SILU ? 1.f : kGelu2 * (1.f + 0.134145f * c * c);
    const float s = logistic(v);
    *grad = s + c * s * (1.f - s) * dv;
    return z * s;
  }
  *grad = 1.f;
  return z;
}

// f with the activation as a compile-time constant (act is wave-uniform).
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  switch (act) {
    case ACT_RELU: f(std::integral_constant<int, ACT_RELU>{}); break;
    case ACT_GELU: f(std::integral_constant<int, ACT_GELU>{}); break;
    case ACT_SILU: f(std::integral_constant<int, ACT_SILU>{}); break;
    default: f(std::integral_constant<int, ACT_NONE>{}); break;
  }
}

}  // namespace ccl
