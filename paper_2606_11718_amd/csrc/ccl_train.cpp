// C ABI of the training operators around the FFN products: the experts'
// products on sorted rows with their gradients, the vocabulary loss and AdamW
// (declarations and contracts: include/ccl.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <exception>
#include <string>
#include <vector>

#include "../../include/ccl.h"
#include "ccl_api.hpp"
#include "host/train.hpp"
#include "kernels/train_kernels.hpp"

using namespace ccl::api;

namespace {

constexpr int64_t kMaxGrid = 0x7fffffff;
constexpr int64_t kMaxElems = (int64_t)1 << 34;   // of a tensor: 2048 a workgroup are fewer than 2^32 threads
constexpr int64_t kMaxTensors = 1 << 20;
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
  if (gated && direction == CCL_GROUPED_FORWARD && s.out * s.w_ld >= (int64_t)1 << 29)
    return fail(CCL_ERR_UNSUPPORTED, "gated: an expert's weight must span less than 2^29 elements");
  // the tiles' numbers are 32-bit, beyond the last by a round of workgroups
  if (ccl::grouped_form(s, rows, direction).tiles > kMaxGrid / 2) return fail(CCL_ERR_UNSUPPORTED, "launch too large");
  *out = s;
  return CCL_OK;
}

ccl_status check_vocab(const ccl_vocab* v, int64_t tokens, bool grad, ccl::VocabShape* out) {
  if (!v) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  if (tokens < 0 || tokens > (int64_t)1 << 30) return fail(CCL_ERR_INVALID_ARG, "tokens must be in 0..2^30");
  if (v->hidden < 1 || v->vocab < 1) return fail(CCL_ERR_INVALID_ARG, "hidden and vocab must be positive");
  if (v->block < 0 || v->block > ccl::kVocabMaxBlock) return fail(CCL_ERR_INVALID_ARG, "block must be in 0..32768");
  if (!std::isfinite(v->scale)) return fail(CCL_ERR_INVALID_ARG, "scale must be finite");
  if (v->hidden % 16 || v->hidden > 1 << 20) return fail(CCL_ERR_UNSUPPORTED, "hidden must be a multiple of 16 up to 2^20");
  if (v->vocab > 1 << 20) return fail(CCL_ERR_UNSUPPORTED, "vocab above 2^20");
  ccl::VocabShape s;
  s.hidden = v->hidden;
  s.vocab = v->vocab;
  s.block = v->block;
  s.scale = v->scale;
  s.w_ld = v->w_ld ? v->w_ld : s.hidden;
  if (s.w_ld < s.hidden || s.w_ld > kMaxLd) return fail(CCL_ERR_INVALID_ARG, "w_ld is smaller than a row of W, or above 2^21");
  if (s.w_ld % 8) return fail(CCL_ERR_MISALIGNED_POINTER, "rows of W must lie whole 16 bytes apart");
  if (tokens) {
    const ccl::VocabForm f = ccl::vocab_form(s, tokens, grad);
    if (ccl::vocab_logits_form(s, f.block, s.vocab, false).tiles > kMaxGrid / 2 ||
        ccl::vocab_dw_form(s, f.block, s.vocab, false).tiles > kMaxGrid / 2 || ccl::vocab_dx_form(s, f.block, false).tiles > kMaxGrid / 2 || (f.block * s.hidden + 1023) / 1024 > kMaxGrid)
      return fail(CCL_ERR_UNSUPPORTED, "launch too large");
  }
  *out = s;
  return CCL_OK;
}

// One buffer of a tensor that a step writes, in bytes.
struct Span {
  uintptr_t from, to;
};
bool overlap(std::vector<Span>& spans) {
  if (!std::is_sorted(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.from < b.from; }))
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
  for (size_t i = 1; i < spans.size(); ++i)
    if (spans[i].from < spans[i - 1].to) return true;
  return false;
}

ccl_status check_adamw_tensor(const ccl_adamw_tensor& t) {
  if (t.n < 0 || t.n > kMaxElems) return fail(CCL_ERR_INVALID_ARG, "a tensor's elements must be in 0..2^34");
  if ((t.param_type != CCL_DT_FP32 && t.param_type != CCL_DT_BF16) || (t.grad_type != CCL_DT_FP32 && t.grad_type != CCL_DT_BF16))
    return fail(CCL_ERR_INVALID_ARG, "param and grad must be fp32 or bf16");
  if (t.moment_bits != 8 && t.moment_bits != 32) return fail(CCL_ERR_INVALID_ARG, "moments have 8 or 32 bits");
  if (!std::isfinite(t.weight_decay)) return fail(CCL_ERR_INVALID_ARG, "weight_decay must be finite");
  if (t.n == 0) return CCL_OK;
  const bool eight = t.moment_bits == 8;
  if (!t.param || !t.grad || !t.exp_avg || !t.exp_avg_sq || (eight && (!t.exp_avg_scale || !t.exp_avg_sq_scale)))
    return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  if (!aligned(t.param, t.param_type == CCL_DT_FP32 ? 4 : 2) || !aligned(t.grad, t.grad_type == CCL_DT_FP32 ? 4 : 2) ||
      (!eight && (!aligned(t.exp_avg, 4) || !aligned(t.exp_avg_sq, 4))) || !aligned(t.copy, 2))
    return fail(CCL_ERR_MISALIGNED_POINTER, "a pointer is not aligned to its elements");
  return CCL_OK;
}

}  // namespace

extern "C" {

ccl_status ccl_grouped_gemm_workspace(const ccl_grouped* grouped, int64_t rows, ccl_grouped_direction direction,
                                      int64_t* workspace_bytes) {
  if (!workspace_bytes) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  ccl::GroupedShape s;
  if (ccl_status st = check_grouped(grouped, rows, direction, &s)) return st;
  *workspace_bytes = ccl::grouped_workspace(s, rows, direction);
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
  if (through && dX == preact && rows > 1 && dx_ld != z_ld)
    return fail(CCL_ERR_INVALID_ARG, "dX in place of preact has its leading dimension");
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

ccl_status ccl_cross_entropy_workspace(const ccl_vocab* vocab, int64_t tokens, int grad, int64_t* workspace_bytes) {
  if (!workspace_bytes) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  if (grad != 0 && grad != 1) return fail(CCL_ERR_INVALID_ARG, "grad must be 0 or 1");
  ccl::VocabShape s;
  if (ccl_status st = check_vocab(vocab, tokens, grad == 1, &s)) return st;
  *workspace_bytes = tokens ? ccl::vocab_form(s, tokens, grad == 1).workspace_bytes : 0;
  return ok();
}

ccl_status ccl_cross_entropy(const ccl_vocab* vocab, int64_t tokens, const void* X, int64_t x_ld, const void* W,
                             const int64_t* targets, float* loss, float* lse, void* workspace, int64_t workspace_bytes,
                             void* stream) {
  ccl::VocabShape s;
  if (ccl_status st = check_vocab(vocab, tokens, false, &s)) return st;
  if (tokens == 0) return ok();
  if (!X || !W || !targets || (!loss && !lse)) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  if (ccl_status st = check_matrix("X", X, x_ld, s.hidden, 8)) return st;
  if (!aligned16(W)) return fail(CCL_ERR_MISALIGNED_POINTER, "W must be 16-byte aligned");
  if (!aligned(targets, 8) || !aligned(loss, 4) || !aligned(lse, 4))
    return fail(CCL_ERR_MISALIGNED_POINTER, "a pointer is not aligned to its elements");
  if (ccl_status st = check_workspace(ccl::vocab_form(s, tokens, false).workspace_bytes, workspace, workspace_bytes)) return st;
  if (ccl_status st = check_device()) return st;
  ccl::VocabCall c;
  c.tokens = tokens;
  c.x = X;
  c.x_ld = x_ld;
  c.w = W;
  c.targets = targets;
  c.loss = loss;
  c.lse = lse;
  return hip_status(ccl::launch_cross_entropy(s, c, workspace, static_cast<hipStream_t>(stream)), "cross entropy launch");
}

ccl_status ccl_cross_entropy_grad(const ccl_vocab* vocab, int64_t tokens, const void* X, int64_t x_ld, const void* W,
                                  const int64_t* targets, const float* dloss, float dloss_scale, float* loss, float* lse,
                                  void* dX, int64_t dx_ld, void* dW, int64_t dw_ld, ccl_dtype dw_type, int accumulate,
                                  void* workspace, int64_t workspace_bytes, void* stream) {
  ccl::VocabShape s;
  if (ccl_status st = check_vocab(vocab, tokens, true, &s)) return st;
  if (dw_type != CCL_DT_BF16 && dw_type != CCL_DT_FP32) return fail(CCL_ERR_INVALID_ARG, "dW must be bf16 or fp32");
  if (accumulate != 0 && accumulate != 1) return fail(CCL_ERR_INVALID_ARG, "accumulate must be 0 or 1");
  if (!dX && !dW) return fail(CCL_ERR_INVALID_ARG, "neither dX nor dW");
  if (dW)
    if (ccl_status st = check_matrix("dW", dW, dw_ld, s.hidden, dw_type == CCL_DT_FP32 ? 4 : 8)) return st;
  if (tokens == 0 && (!dW || accumulate)) return ok();
  if (tokens && (!X || !W || !targets)) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  if (tokens) {
    if (ccl_status st = check_matrix("X", X, x_ld, s.hidden, 8)) return st;
    if (dX)
      if (ccl_status st = check_matrix("dX", dX, dx_ld, s.hidden, 8)) return st;
    if (!aligned16(W)) return fail(CCL_ERR_MISALIGNED_POINTER, "W must be 16-byte aligned");
    if (!aligned(targets, 8) || !aligned(dloss, 4) || !aligned(loss, 4) || !aligned(lse, 4))
      return fail(CCL_ERR_MISALIGNED_POINTER, "a pointer is not aligned to its elements");
    if (ccl_status st = check_workspace(ccl::vocab_form(s, tokens, true).workspace_bytes, workspace, workspace_bytes)) return st;
  }
  if (ccl_status st = check_device()) return st;
  ccl::VocabCall c;
  c.tokens = tokens;
  c.x = X;
  c.x_ld = x_ld;
  c.w = W;
  c.targets = targets;
  c.loss = loss;
  c.lse = lse;
  c.grad = true;
  c.dloss = dloss;
  c.dloss_scale = dloss_scale;
  c.dx = dX;
  c.dx_ld = dx_ld;
  c.dw = dW;
  c.dw_ld = dw_ld;
  c.dw_f32 = dw_type == CCL_DT_FP32;
  c.accumulate = accumulate == 1;
  return hip_status(ccl::launch_cross_entropy(s, c, workspace, static_cast<hipStream_t>(stream)), "cross entropy gradient launch");
}

ccl_status ccl_adamw_step(const ccl_adamw* adamw, const ccl_adamw_tensor* tensors, int64_t count, void* stream) try {
  if (!adamw || (count > 0 && !tensors)) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  if (count < 0 || count > kMaxTensors) return fail(CCL_ERR_INVALID_ARG, "count must be in 0..2^20");
  if (!std::isfinite(adamw->lr) || !(adamw->beta1 >= 0 && adamw->beta1 < 1) || !(adamw->beta2 >= 0 && adamw->beta2 < 1) ||
      !(adamw->eps >= 0) || !std::isfinite(adamw->eps))
    return fail(CCL_ERR_INVALID_ARG, "lr must be finite, the betas in [0, 1), eps finite and not negative");
  if (!adamw->step_ptr && adamw->step < 1) return fail(CCL_ERR_INVALID_ARG, "step counts from 1");
  if (!aligned(adamw->step_ptr, 8) || !aligned(adamw->lr_ptr, 4) || !aligned(adamw->grad_scale, 4))
    return fail(CCL_ERR_MISALIGNED_POINTER, "a pointer is not aligned to its elements");
  std::vector<ccl::AdamwTensor> kinds[8];
  std::vector<Span> written;
  written.reserve(6 * (size_t)count);
  for (int pass = 0; pass < 6; ++pass)      // one kind of buffer after the other: most callers' are in order
    for (int64_t i = 0; i < count; ++i) {
      const ccl_adamw_tensor& t = tensors[i];
      if (pass == 0)
        if (ccl_status s = check_adamw_tensor(t)) return s;
      if (t.n == 0) continue;
      const int64_t moment = t.moment_bits == 8 ? t.n : 4 * t.n;
      const int64_t blocks = t.moment_bits == 8 ? (t.n + ccl::kAdamwBlock - 1) / ccl::kAdamwBlock : 0;
      const auto add = [&](const void* p, int64_t bytes) {
        if (p) written.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes});
      };
      if (pass == 0) add(t.param, t.param_type == CCL_DT_FP32 ? 4 * t.n : 2 * t.n);
      if (pass == 1) add(t.exp_avg, moment);
      if (pass == 2) add(t.exp_avg_sq, moment);
      if (pass == 3) add(t.copy, 2 * t.n);
      if (pass == 4 && blocks) add(t.exp_avg_scale, blocks);
      if (pass == 5 && blocks) add(t.exp_avg_sq_scale, blocks);
    }
  if (overlap(written)) return fail(CCL_ERR_INVALID_ARG, "buffers that the step writes overlap (a tensor given twice?)");
  if (written.empty()) return ok();
  if (ccl_status s = check_device()) return s;
  for (int64_t i = 0; i < count; ++i) {
    const ccl_adamw_tensor& t = tensors[i];
    if (t.n == 0) continue;
    ccl::AdamwTensor k{t.param, t.grad, t.exp_avg, t.exp_avg_sq, t.exp_avg_scale, t.exp_avg_sq_scale,
                       static_cast<uint16_t*>(t.copy), t.n, t.weight_decay};
    kinds[(t.param_type == CCL_DT_BF16) * 4 + (t.grad_type == CCL_DT_BF16) * 2 + (t.moment_bits == 8)].push_back(k);
  }
  ccl::AdamwStep a;
  a.lr = adamw->lr;
  a.beta1 = adamw->beta1;
  a.beta2 = adamw->beta2;
  a.eps = adamw->eps;
  a.step = adamw->step;
  a.step_ptr = adamw->step_ptr;
  a.lr_ptr = adamw->lr_ptr;
  a.grad_scale = adamw->grad_scale;
  for (int k = 0; k < 8; ++k)
    if (!kinds[k].empty())
      if (hipError_t e = ccl::launch_adamw(a, kinds[k].data(), (int64_t)kinds[k].size(), k & 4, k & 2, k & 1,
                                           static_cast<hipStream_t>(stream)))
        return hip_status(e, "adamw launch");
  return ok();
} catch (const std::exception& e) {
  return fail(CCL_ERR_HIP, e.what());
}

ccl_status ccl_adamw_moments(int64_t n, const uint8_t* exp_avg, const uint8_t* exp_avg_scale, const uint8_t* exp_avg_sq,
                             const uint8_t* exp_avg_sq_scale, void* m, void* v, ccl_dtype type, void* stream) {
  if (n < 0 || n > kMaxElems) return fail(CCL_ERR_INVALID_ARG, "n must be in 0..2^34");
  if (type != CCL_DT_FP32 && type != CCL_DT_BF16) return fail(CCL_ERR_INVALID_ARG, "the values are fp32 or bf16");
  if (n == 0 || (!m && !v)) return ok();
  if ((m && (!exp_avg || !exp_avg_scale)) || (v && (!exp_avg_sq || !exp_avg_sq_scale)))
    return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  if (!aligned(m, type == CCL_DT_FP32 ? 4 : 2) || !aligned(v, type == CCL_DT_FP32 ? 4 : 2))
    return fail(CCL_ERR_MISALIGNED_POINTER, "a pointer is not aligned to its elements");
  if (ccl_status s = check_device()) return s;
  return hip_status(ccl::launch_adamw_moments(n, exp_avg, exp_avg_scale, exp_avg_sq, exp_avg_sq_scale, m, v,
                                              type == CCL_DT_BF16, static_cast<hipStream_t>(stream)),
                    "adamw moments launch");
}

}  // extern "C"
