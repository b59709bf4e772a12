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

}  // namespace ccl
