// Activations of the FFN operators and their derivatives, in fp32.
//
//   relu(z) = max(z, 0)              silu(z) = z s(z), s the logistic function
//   gelu(z) = z s(2u), u = sqrt(2/pi) (z + 0.044715 z^3)   (the tanh form:
//             (1 + tanh u) / 2 = s(2u))
//
// s(x) = 1 / (1 + 2^(-x log2 e)) is one v_exp_f32 and one v_rcp_f32 (1 ulp
// each), so an activation is within a few ulp of fp32 wherever it is not
// tiny; a large negative x gives 1 / inf = 0. NaN stays NaN. s is formed at z
// clamped to +-100, where it is 0 or 1 to the last bit: beyond 2^64, z^2 is
// infinite and SiLU's zero coefficient of it would make a NaN.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "../host/plan.hpp"

namespace ccl {

// 1 / (1 + 2^x), s(v) for x = -v log2 e.
__device__ __forceinline__ float logistic2(float x) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x));
}

constexpr float kLog2e = 1.44269504089f;
constexpr float kGelu2 = 1.59576912161f;   // 2 sqrt(2/pi)

// GELU and SiLU are one formula, z s(z (k0 + k1 z^2)): SiLU has k0 = 1, k1 = 0.
enum ActClass { ACT_CLASS_NONE, ACT_CLASS_RELU, ACT_CLASS_SMOOTH };
struct ActCoef {
  float k0, k1;
};
__device__ __forceinline__ ActCoef act_coef(int act) {
  return act == ACT_GELU ? ActCoef{kGelu2, 0.044715f * kGelu2} : ActCoef{1.f, 0.f};
}

template <int CLASS>
__device__ __forceinline__ float act_value(ActCoef k, float z) {
  if constexpr (CLASS == ACT_CLASS_RELU) return z < 0.f ? 0.f : z;
  if constexpr (CLASS == ACT_CLASS_SMOOTH) {
    const float c = __builtin_amdgcn_fmed3f(z, -100.f, 100.f);
    return z * logistic2(c * __builtin_fmaf(-kLog2e * k.k1, c * c, -kLog2e * k.k0));
  }
  return z;
}

// Value and derivative. The derivative is formed at z clamped to +-100, where
// both functions are 0 or z to the last bit: beyond, its factors would meet as
// 0 * inf. With s = s(v): s' = s (1 - s) v'.
template <int CLASS>
__device__ __forceinline__ float act_value_grad(ActCoef k, float z, float* grad) {
  if constexpr (CLASS == ACT_CLASS_RELU) {
    *grad = z > 0.f ? 1.f : (z <= 0.f ? 0.f : z);   // 0 at 0, NaN at NaN
    return z < 0.f ? 0.f : z;
  }
  if constexpr (CLASS == ACT_CLASS_SMOOTH) {
    const float c = z > 100.f ? 100.f : (z < -100.f ? -100.f : z);
    const float s = logistic2(c * __builtin_fmaf(-kLog2e * k.k1, c * c, -kLog2e * k.k0));
    *grad = __builtin_fmaf(c * s * (1.f - s), __builtin_fmaf(3.f * k.k1, c * c, k.k0), s);
    return z * s;
  }
  *grad = 1.f;
  return z;
}

// f with the activation's class as a compile-time constant (act is uniform).
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  if (act == ACT_NONE) f(std::integral_constant<int, ACT_CLASS_NONE>{});
  else if (act == ACT_RELU) f(std::integral_constant<int, ACT_CLASS_RELU>{});
  else f(std::integral_constant<int, ACT_CLASS_SMOOTH>{});
}

}  // namespace ccl
