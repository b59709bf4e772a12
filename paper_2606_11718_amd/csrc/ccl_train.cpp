// C ABI of the training operators around the FFN products: the experts'
// products on sorted rows with their gradients (declarations and contracts:
// include/ccl.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <string>

#include "../../include/ccl.h"
#include "ccl_api.hpp"
#include "host/train.hpp"
#include "kernels/train_kernels.hpp"

using namespace ccl::api;

namespace {

constexpr int64_t kMaxGrid = 0x7fffffff;
constexpr int64_t kMaxLd = (int64_t)1 << 21;      // 256 rows stay within 31-bit byte offsets
constexpr int64_t kMaxStride = (int64_t)1 << 48;

ccl_status check_workspace(int64_t need, const void* workspace, int64_t bytes) {
  if (need == 0) return CCL_OK;
  if (!workspace) return fail(CCL_ERR_INVALID_ARG, "NULL workspace");
  if (bytes < need) return fail(CCL_ERR_INVALID_ARG, "workspace smaller than the " + std::to_string(need) + " bytes reported");
  if (!aligned16(workspace)) return fail(CCL_ERR_MISALIGNED_POINTER, "the workspace must be 16-byte aligned");
  return CCL_OK;
}

// A matrix of rows of `cols` elements, `per` of them 16 bytes.
ccl_status check_matrix(const char* name, const void* p, int64_t ld, int64_t cols, int64_t per) {
  if (ld < cols || ld > kMaxLd)
    return fail(CCL_ERR_INVALID_ARG, std::string(name) + ": a leading dimension smaller than its row, or above 2^21");
  if (!aligned16(p) || ld % per)
    return fail(CCL_ERR_MISALIGNED_POINTER, std::string(name) + " (and its rows) must be 16-byte aligned");
  return CCL_OK;
}

ccl_status check_grouped(const ccl_grouped* g, int64_t rows, int direction, ccl::GroupedShape* out) {
  if (!g) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  if (direction < CCL_GROUPED_FORWARD || direction > CCL_GROUPED_WGRAD) return fail(CCL_ERR_INVALID_ARG, "unknown direction");
  if (rows < 0 || rows > (int64_t)1 << 30) return fail(CCL_ERR_INVALID_ARG, "rows must be in 0..2^30");
  if (g->in_features < 1 || g->out_features < 1) return fail(CCL_ERR_INVALID_ARG, "in_features and out_features must be positive");
  if (g->experts < 1 || g->experts > ccl::kGroupedMaxExperts) return fail(CCL_ERR_INVALID_ARG, "experts must be in 1..512");
  if (g->activation < CCL_ACT_NONE || g->activation > CCL_ACT_SILU) return fail(CCL_ERR_INVALID_ARG, "unknown activation");
  if (g->gated != 0 && g->gated != 1) return fail(CCL_ERR_INVALID_ARG, "gated must be 0 or 1");
  constexpr int64_t kMaxSide = 1 << 20;
  if (g->in_features % 16 || g->out_features % 16 || g->in_features > kMaxSide || g->out_features > kMaxSide)
    return fail(CCL_ERR_UNSUPPORTED, "in_features and out_features must be multiples of 16 up to 2^20");
  const bool gated = g->gated == 1;
  if (gated && direction == CCL_GROUPED_FORWARD && g->out_features % 32)
    return fail(CCL_ERR_UNSUPPORTED, "gated: out_features (gate and up rows) must be a multiple of 32");
  ccl::GroupedShape s;
  s.in = g->in_features;
  s.out = g->out_features;
  s.experts = g->experts;
  s.act = g->activation;
  s.gated = gated;
  s.w_ld = g->w_ld ? g->w_ld : s.in;
  if (s.w_ld < s.in || s.w_ld > kMaxLd)
    return fail(CCL_ERR_INVALID_ARG, "w_ld is smaller than a weight's row, or above 2^21");
  s.w_stride = g->w_stride ? g->w_stride : s.out * s.w_ld;
  // an expert's last row need not be followed by a gap
  if (s.w_stride < (s.out - 1) * s.w_ld + s.in || s.w_stride > kMaxStride)
    return fail(CCL_ERR_INVALID_ARG, "experts' weights overlap, or lie more than 2^48 elements apart");
  if (s.w_ld % 8 || s.w_stride % 8)
    return fail(CCL_ERR_MISALIGNED_POINTER, "weight rows and experts must lie whole 16 bytes apart");
  if (gated && direction == CCL_GROUPED_FORWARD && s.out * s.w_ld >= (int64_t)1 << 30)
    return fail(CCL_ERR_UNSUPPORTED, "gated: an expert's weight must span less than 2^30 elements");
  if (ccl::grouped_form(s, rows, direction).workgroups > kMaxGrid) return fail(CCL_ERR_UNSUPPORTED, "launch too large");
  *out = s;
  return CCL_OK;
}

}  // namespace

extern "C" {

ccl_status ccl_grouped_gemm_workspace(const ccl_grouped* grouped, int64_t rows, ccl_grouped_direction direction,
                                      int64_t* workspace_bytes) {
  if (!workspace_bytes) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  ccl::GroupedShape s;
  if (ccl_status st = check_grouped(grouped, rows, direction, &s)) return st;
  *workspace_bytes = rows ? ccl::grouped_form(s, rows, direction).workspace_bytes : 0;
  return ok();
}

ccl_status ccl_grouped_gemm(const ccl_grouped* grouped, int64_t rows, const int32_t* ends, const void* X, int64_t x_ld,
                            const void* W, void* Y, int64_t y_ld, void* preact, int64_t z_ld, void* workspace,
                            int64_t workspace_bytes, void* stream) {
  ccl::GroupedShape s;
  if (ccl_status st = check_grouped(grouped, rows, CCL_GROUPED_FORWARD, &s)) return st;
  if (rows == 0) return ok();
  if (!ends || !X || !W || !Y) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  if (!aligned(ends, 4)) return fail(CCL_ERR_MISALIGNED_POINTER, "ends must be 4-byte aligned");
  if (!aligned16(W)) return fail(CCL_ERR_MISALIGNED_POINTER, "W must be 16-byte aligned");
  if (ccl_status st = check_matrix("X", X, x_ld, s.in, 8)) return st;
  if (ccl_status st = check_matrix("Y", Y, y_ld, s.gated ? s.out / 2 : s.out, 8)) return st;
  if (preact)
    if (ccl_status st = check_matrix("preact", preact, z_ld, s.out, 8)) return st;
  if (ccl_status st = check_workspace(ccl::grouped_form(s, rows, CCL_GROUPED_FORWARD).workspace_bytes, workspace, workspace_bytes))
    return st;
  if (ccl_status st = check_device()) return st;
  ccl::GroupedCall c;
  c.rows = rows;
  c.ends = ends;
  c.a = X;
  c.a_ld = x_ld;
  c.b = W;
  c.out = Y;
  c.out_ld = y_ld;
  c.z = preact;
  c.z_ld = z_ld;
  return hip_status(ccl::launch_grouped(s, c, CCL_GROUPED_FORWARD, workspace, static_cast<hipStream_t>(stream)),
                    "grouped gemm launch");
}

ccl_status ccl_grouped_gemm_grad(const ccl_grouped* grouped, int64_t rows, const int32_t* ends, const void* dY,
                                 int64_t dy_ld, const void* W, void* dX, int64_t dx_ld, const void* preact, int64_t z_ld,
                                 void* workspace, int64_t workspace_bytes, void* stream) {
  ccl::GroupedShape s;
  if (ccl_status st = check_grouped(grouped, rows, CCL_GROUPED_GRAD, &s)) return st;
  if (rows == 0) return ok();
  if (!ends || !dY || !W || !dX) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  const bool through = s.act != CCL_ACT_NONE || s.gated;
  if (through && !preact) return fail(CCL_ERR_INVALID_ARG, "NULL preact");
  const int64_t wide = s.gated ? 2 * s.in : s.in;
  if (!aligned(ends, 4)) return fail(CCL_ERR_MISALIGNED_POINTER, "ends must be 4-byte aligned");
  if (!aligned16(W)) return fail(CCL_ERR_MISALIGNED_POINTER, "W must be 16-byte aligned");
  if (ccl_status st = check_matrix("dY", dY, dy_ld, s.out, 8)) return st;
  if (ccl_status st = check_matrix("dX", dX, dx_ld, wide, 8)) return st;
  if (through)
    if (ccl_status st = check_matrix("preact", preact, z_ld, wide, 8)) return st;
  if (ccl_status st = check_workspace(ccl::grouped_form(s, rows, CCL_GROUPED_GRAD).workspace_bytes, workspace, workspace_bytes))
    return st;
  if (ccl_status st = check_device()) return st;
  ccl::GroupedCall c;
  c.rows = rows;
  c.ends = ends;
  c.a = dY;
  c.a_ld = dy_ld;
  c.b = W;
  c.out = dX;
  c.out_ld = dx_ld;
  c.z = const_cast<void*>(preact);
  c.z_ld = z_ld;
  return hip_status(ccl::launch_grouped(s, c, CCL_GROUPED_GRAD, workspace, static_cast<hipStream_t>(stream)),
                    "grouped gradient gemm launch");
}

ccl_status ccl_grouped_gemm_wgrad(const ccl_grouped* grouped, int64_t rows, const int32_t* ends, const void* dY,
                                  int64_t dy_ld, const void* X, int64_t x_ld, void* dW, ccl_dtype dw_type, int accumulate,
                                  void* workspace, int64_t workspace_bytes, void* stream) {
  ccl::GroupedShape s;
  if (ccl_status st = check_grouped(grouped, rows, CCL_GROUPED_WGRAD, &s)) return st;
  if (dw_type != CCL_DT_BF16 && dw_type != CCL_DT_FP32) return fail(CCL_ERR_INVALID_ARG, "dW must be bf16 or fp32");
  if (accumulate != 0 && accumulate != 1) return fail(CCL_ERR_INVALID_ARG, "accumulate must be 0 or 1");
  if (rows == 0 && accumulate) return ok();
  if (!ends || (rows && (!dY || !X)) || !dW) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  if (!aligned(ends, 4)) return fail(CCL_ERR_MISALIGNED_POINTER, "ends must be 4-byte aligned");
  if (!aligned16(dW)) return fail(CCL_ERR_MISALIGNED_POINTER, "dW must be 16-byte aligned");
  if (ccl_status st = check_matrix("dY", dY, dy_ld, s.out, 8)) return st;
  if (ccl_status st = check_matrix("X", X, x_ld, s.in, 8)) return st;
  if (ccl_status st = check_workspace(rows ? ccl::grouped_form(s, rows, CCL_GROUPED_WGRAD).workspace_bytes : 0, workspace,
                                      workspace_bytes))
    return st;
  if (ccl_status st = check_device()) return st;
  ccl::GroupedCall c;
  c.rows = rows;
  c.ends = ends;
  c.a = dY;
  c.a_ld = dy_ld;
  c.b = X;
  c.b_ld = x_ld;
  c.out = dW;
  c.f32 = dw_type == CCL_DT_FP32;
  c.accumulate = accumulate == 1;
  return hip_status(ccl::launch_grouped(s, c, CCL_GROUPED_WGRAD, workspace, static_cast<hipStream_t>(stream)),
                    "grouped weight gradient launch");
}

}  // extern "C"
