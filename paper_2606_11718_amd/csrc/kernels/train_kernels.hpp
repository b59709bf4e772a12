// Kernel launchers of the training operators (device side: grouped.hip,
// cross_entropy.hip, adamw.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../host/train.hpp"

namespace ccl {

// One call of ccl_grouped_gemm (a = X, b = W, out = Y), _grad (a = dY, b = W,
// out = dX) or _wgrad (a = dY, b = X, out = dW); ws: grouped_form's workspace.
struct GroupedCall {
  int64_t rows = 0;
  const int32_t* ends = nullptr;
  const void *a = nullptr, *b = nullptr;
  void *out = nullptr, *z = nullptr;
  int64_t a_ld = 0, b_ld = 0, out_ld = 0, z_ld = 0;
  bool f32 = false, accumulate = false;
};
hipError_t launch_grouped(const GroupedShape& s, const GroupedCall& c, int direction, void* ws, hipStream_t stream);

// One call of ccl_cross_entropy (grad false) or _grad; ws: vocab_form's workspace.
struct VocabCall {
  int64_t tokens = 0;
  const void *x = nullptr, *w = nullptr;
  int64_t x_ld = 0;
  const int64_t* targets = nullptr;
  float *loss = nullptr, *lse = nullptr;
  bool grad = false;
  const float* dloss = nullptr;
  float dloss_scale = 1.f;
  void *dx = nullptr, *dw = nullptr;
  int64_t dx_ld = 0, dw_ld = 0;
  bool dw_f32 = false, accumulate = false;
};
hipError_t launch_cross_entropy(const VocabShape& s, const VocabCall& c, void* ws, hipStream_t stream);

// One tensor of a ccl_adamw_step: 16-bit or 32-bit param and grad, moments of 32
// or 8 bits (then with their scales).
struct AdamwTensor {
  void* param;
  const void* grad;
  void *m, *v;
  uint8_t *m_scale, *v_scale;
  uint16_t* copy;
  int64_t n;
  float weight_decay;
};
struct AdamwStep {
  double lr = 0, beta1 = 0, beta2 = 0, eps = 0;
  int64_t step = 0;
  const int64_t* step_ptr = nullptr;
  const float *lr_ptr = nullptr, *grad_scale = nullptr;
};
// The tensors of one kind, count of them.
hipError_t launch_adamw(const AdamwStep& a, const AdamwTensor* tensors, int64_t count, bool p_bf16, bool g_bf16, bool bits8,
                        hipStream_t stream);
hipError_t launch_adamw_moments(int64_t n, const uint8_t* m, const uint8_t* m_scale, const uint8_t* v, const uint8_t* v_scale,
                                void* m_out, void* v_out, bool bf16, hipStream_t stream);

}  // namespace ccl
