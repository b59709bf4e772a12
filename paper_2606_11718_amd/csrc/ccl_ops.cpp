// C ABI of the FFN operators around the GEMM (declarations and contracts:
// include/ccl.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "../../include/ccl.h"
#include "ccl_api.hpp"
#include "host/plan.hpp"
#include "kernels/kernels.hpp"

using namespace ccl::api;

namespace {

constexpr int64_t kMaxGrid = 0x7fffffff;

bool valid_layout(int l) { return l == CCL_LAYOUT_CCL || l == CCL_LAYOUT_ROWMAJOR; }

// What both directions check of the plan, the epilogue's fields and the
// launch; on CCL_OK *form is what to launch.
ccl_status check_fused(ccl_plan_t plan, int layout, int activation, int gated, int64_t rows, int splits, bool grad,
                       bool dbias, ccl::FusedForm* form) {
  const ccl::Plan& p = plan->plan;
  if (!valid_layout(layout)) return fail(CCL_ERR_INVALID_ARG, "layout must be CCL_LAYOUT_CCL or CCL_LAYOUT_ROWMAJOR");
  if (!ccl::valid_act(activation)) return fail(CCL_ERR_INVALID_ARG, "unknown activation");
  if (gated != 0 && gated != 1) return fail(CCL_ERR_INVALID_ARG, "gated must be 0 or 1");
  if (rows < 0 || rows > p.M) return fail(CCL_ERR_INVALID_ARG, "rows must be in 0..M");
  if (!p.gemm.supported) return fail(CCL_ERR_UNSUPPORTED, p.gemm.why_unsupported);
  if (p.c_type != ccl::DT_BF16) return fail(CCL_ERR_UNSUPPORTED, "the fused epilogues write a bf16 C");
  if (splits < 1 || splits > ccl::kMaxSplits) return fail(CCL_ERR_INVALID_ARG, "splits must be in 1..16");
  if (ccl::splitk_workgroups(p, splits) > kMaxGrid || ccl::splitk_reduce_workgroups(p) > kMaxGrid)
    return fail(CCL_ERR_UNSUPPORTED, "grid exceeds the launch limit");
  if (grad && gated && 2 * p.N > kMaxGrid) return fail(CCL_ERR_UNSUPPORTED, "2 N exceeds 31 bits");
  *form = ccl::fused_form(p, layout == CCL_LAYOUT_ROWMAJOR, splits, grad, gated == 1, dbias, rows, 0);
  if (!offsets_fit(p, form->a, form->b)) return fail(CCL_ERR_UNSUPPORTED, "rows too long for 32-bit in-tile offsets");
  return CCL_OK;
}

ccl_status check_workspace(int64_t need, const void* workspace, int64_t bytes) {
  if (need == 0) return CCL_OK;
  if (!workspace) return fail(CCL_ERR_INVALID_ARG, "NULL workspace");
  if (bytes < need) return fail(CCL_ERR_INVALID_ARG, "workspace smaller than the " + std::to_string(need) + " bytes reported");
  if (!aligned16(workspace)) return fail(CCL_ERR_MISALIGNED_POINTER, "the workspace must be 16-byte aligned");
  return CCL_OK;
}

// The checked shape of a layer for a number of tokens.
ccl_status check_moe(const ccl_moe* m, int64_t tokens, ccl::MoeShape* out) {
  if (!m) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  if (tokens < 0 || tokens > ccl::kMoeMaxTokens) return fail(CCL_ERR_INVALID_ARG, "tokens must be in 0..64");
  if (m->hidden < 1 || m->ffn < 1) return fail(CCL_ERR_INVALID_ARG, "hidden and ffn must be positive");
  if (m->experts < 1 || m->experts > ccl::kMoeMaxExperts) return fail(CCL_ERR_INVALID_ARG, "experts must be in 1..512");
  if (m->top_k < 1 || m->top_k > ccl::kMoeMaxTopK || m->top_k > m->experts)
    return fail(CCL_ERR_INVALID_ARG, "top_k must be in 1..16 and at most the experts");
  if (!ccl::valid_act(m->activation)) return fail(CCL_ERR_INVALID_ARG, "unknown activation");
  if (m->normalize != 0 && m->normalize != 1) return fail(CCL_ERR_INVALID_ARG, "normalize must be 0 or 1");
  if (m->weight_type != CCL_DT_BF16 && m->weight_type != CCL_DT_FP8_E4M3)
    return fail(CCL_ERR_INVALID_ARG, "weights must be bf16 or fp8 E4M3");
  constexpr int64_t kMaxSide = 1 << 22, kMaxStride = (int64_t)1 << 48;
  if (m->hidden % 16 || m->ffn % 16 || m->hidden > kMaxSide || m->ffn > kMaxSide)
    return fail(CCL_ERR_UNSUPPORTED, "hidden and ffn must be multiples of 16 up to 2^22");
  ccl::MoeShape s;
  s.hidden = m->hidden;
  s.ffn = m->ffn;
  s.experts = m->experts;
  s.top_k = m->top_k;
  s.act = m->activation;
  s.normalize = m->normalize == 1;
  s.fp8 = m->weight_type == CCL_DT_FP8_E4M3;
  const int64_t per = s.fp8 ? 16 : 8;
  s.gu_ld = m->gate_up_ld ? m->gate_up_ld : m->hidden;
  s.down_ld = m->down_ld ? m->down_ld : m->ffn;
  if (s.gu_ld < m->hidden || s.down_ld < m->ffn || s.gu_ld > kMaxSide || s.down_ld > kMaxSide)
    return fail(CCL_ERR_INVALID_ARG, "a weight's leading dimension is smaller than its rows, or above 2^22");
  s.gu_stride = m->gate_up_stride ? m->gate_up_stride : 2 * m->ffn * s.gu_ld;
  s.down_stride = m->down_stride ? m->down_stride : m->hidden * s.down_ld;
  // an expert's last row need not be followed by a gap
  if (s.gu_stride < (2 * m->ffn - 1) * s.gu_ld + m->hidden || s.down_stride < (m->hidden - 1) * s.down_ld + m->ffn ||
      s.gu_stride > kMaxStride || s.down_stride > kMaxStride)
    return fail(CCL_ERR_INVALID_ARG, "experts overlap, or lie more than 2^48 elements apart");
  if (s.gu_ld % per || s.gu_stride % per || s.down_ld % per || s.down_stride % per)
    return fail(CCL_ERR_MISALIGNED_POINTER, "weight rows and experts must lie whole 16 bytes apart");
  if (tokens * s.top_k * s.ffn >= (int64_t)1 << 29)
    return fail(CCL_ERR_UNSUPPORTED, "tokens * top_k * ffn must be below 2^29");
  const ccl::MoeForm f = ccl::moe_form(s, tokens);
  if (f.up_workgroups > kMaxGrid || (int64_t)f.down_groups * f.splits > kMaxGrid)
    return fail(CCL_ERR_UNSUPPORTED, "launch too large");
  *out = s;
  return CCL_OK;
}

ccl_status check_ortho(int64_t batch, int64_t rows, int64_t cols) {
  if (batch < 0 || rows < 0 || cols < 0) return fail(CCL_ERR_INVALID_ARG, "negative size");
  if (rows > 65536 || cols > 65536) return fail(CCL_ERR_UNSUPPORTED, "a side above 65536");
  if (batch > kMaxGrid) return fail(CCL_ERR_UNSUPPORTED, "launch too large");
  const ccl::OrthoForm f = ccl::ortho_form({batch, rows, cols});
  if (f.x_elems >= (int64_t)1 << 30) return fail(CCL_ERR_UNSUPPORTED, "a matrix of 2^30 padded elements or more");
  // the launches of most workgroups: 64x64 pieces, elements without steps, 128x128 tiles
  if (batch * ((rows * cols + 255) / 256) > kMaxGrid || batch * (f.x_elems / 4096) > kMaxGrid ||
      batch * f.chunks > kMaxGrid)
    return fail(CCL_ERR_UNSUPPORTED, "launch too large");
  return CCL_OK;
}

}  // namespace

extern "C" {

ccl_status ccl_plan_matrix_layout(ccl_plan_t plan, int64_t cols, ccl_layout* out) {
  if (!plan || !out) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  if (cols < 1 || cols > kMaxGrid || cols % plan->plan.Gc != 0)
    return fail(CCL_ERR_INVALID_ARG, "cols must be a positive multiple of the grid's columns below 2^31");
  const ccl::Layout l = ccl::matrix_layout(plan->plan, cols);
  out->rows = l.rows;
  out->cols = l.cols;
  out->grid_r = l.grid_r;
  out->grid_c = l.grid_c;
  out->block_rows = l.block_rows;
  out->block_cols = l.block_cols;
  out->strip_bytes = l.strip_bytes;
  out->strip_stride_bytes = l.strip_stride_bytes;
  out->total_bytes = l.total_bytes;
  out->elem_bytes = l.elem_bytes;
  return ok();
}

ccl_status ccl_gemm_fused_workspace(ccl_plan_t plan, ccl_operand_layout layout, int* splits,
                                    int64_t* workspace_bytes) {
  if (!plan || !splits || !workspace_bytes) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  if (*splits < 0 || *splits > ccl::kMaxSplits)
    return fail(CCL_ERR_INVALID_ARG, "splits must be 0 (choose) or in 1..16");
  const int s = *splits == 0 ? ccl::recommended_splits(plan->plan) : *splits;
  ccl::FusedForm f;
  if (ccl_status st = check_fused(plan, layout, CCL_ACT_NONE, 0, 0, s, false, false, &f)) return st;
  *splits = f.gemm.splits;
  *workspace_bytes = f.workspace_bytes;
  return ok();
}

ccl_status ccl_gemm_fused(ccl_plan_t plan, const ccl_epilogue* e, const void* A, const void* B, void* C,
                          int splits, void* workspace, int64_t workspace_bytes, void* stream) {
  if (!plan || !e || !A || !B || !C) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  ccl::FusedForm f;
  if (ccl_status s = check_fused(plan, e->layout, e->activation, e->gated, e->rows, splits, false, false, &f)) return s;
  if (e->bias && e->bias_type != CCL_DT_FP32 && e->bias_type != CCL_DT_BF16)
    return fail(CCL_ERR_INVALID_ARG, "the bias must be fp32 or bf16");
  if (!aligned16(A) || !aligned16(B) || !aligned16(C) || !aligned16(e->bias) || !aligned16(e->residual) ||
      !aligned16(e->preact))
    return fail(CCL_ERR_MISALIGNED_POINTER, "A, B, C, bias, residual and preact must be 16-byte aligned");
  if (ccl_status s = check_workspace(f.workspace_bytes, workspace, workspace_bytes)) return s;
  if (ccl_status s = check_device()) return s;
  ccl::FusedCall c;
  c.A = A;
  c.B = B;
  c.C = C;
  c.bias = e->bias;
  c.bias_f32 = e->bias_type == CCL_DT_FP32;
  c.R = e->residual;
  c.Zout = e->preact;
  c.rowmajor = e->layout == CCL_LAYOUT_ROWMAJOR;
  c.gated = e->gated == 1;
  c.act = e->activation;
  c.alpha = e->alpha;
  c.beta = e->beta;
  c.rows = e->rows;
  return hip_status(ccl::launch_gemm_fused(plan->plan, c, splits, workspace, static_cast<hipStream_t>(stream)),
                    "fused gemm launch");
}

ccl_status ccl_gemm_fused_grad_workspace(ccl_plan_t plan, ccl_operand_layout layout, int gated, int dbias,
                                         int64_t* workspace_bytes) {
  if (!plan || !workspace_bytes) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  if (dbias != 0 && dbias != 1) return fail(CCL_ERR_INVALID_ARG, "dbias must be 0 or 1");
  ccl::FusedForm f;
  if (ccl_status s = check_fused(plan, layout, CCL_ACT_NONE, gated, 0, ccl::kMaxSplits, true, dbias == 1, &f)) return s;
  *workspace_bytes = f.workspace_bytes;
  return ok();
}

ccl_status ccl_gemm_fused_grad(ccl_plan_t plan, const ccl_epilogue_grad* e, const void* A, const void* B, void* dZ,
                               void* workspace, int64_t workspace_bytes, void* stream) {
  if (!plan || !e || !A || !B || !dZ) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  ccl::FusedForm f;
  if (ccl_status s = check_fused(plan, e->layout, e->activation, e->gated, e->rows, ccl::kMaxSplits, true,
                                 e->dbias != nullptr, &f))
    return s;
  const bool linear = e->activation == CCL_ACT_NONE && e->gated == 0;
  if (!e->preact && !linear) return fail(CCL_ERR_INVALID_ARG, "NULL preact");
  if (!aligned16(A) || !aligned16(B) || !aligned16(dZ) || !aligned16(e->preact) || !aligned16(e->dbias))
    return fail(CCL_ERR_MISALIGNED_POINTER, "A, B, dZ, preact and dbias must be 16-byte aligned");
  if (ccl_status s = check_workspace(f.workspace_bytes, workspace, workspace_bytes)) return s;
  if (ccl_status s = check_device()) return s;
  ccl::FusedCall c;
  c.A = A;
  c.B = B;
  c.C = dZ;
  c.Zin = linear ? nullptr : e->preact;
  c.dbias = e->dbias;
  c.rowmajor = e->layout == CCL_LAYOUT_ROWMAJOR;
  c.grad = true;
  c.gated = e->gated == 1;
  c.act = e->activation;
  c.alpha = e->alpha;
  c.rows = e->rows;
  return hip_status(ccl::launch_gemm_fused(plan->plan, c, ccl::kMaxSplits, workspace, static_cast<hipStream_t>(stream)),
                    "fused gradient gemm launch");
}

ccl_status ccl_moe_workspace(const ccl_moe* moe, int64_t tokens, int64_t* workspace_bytes) {
  if (!workspace_bytes) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  ccl::MoeShape s;
  if (ccl_status st = check_moe(moe, tokens, &s)) return st;
  // a smaller number of tokens may need more (it may be launched otherwise)
  int64_t most = 0;
  for (int64_t t = 0; t <= tokens; ++t) most = std::max(most, ccl::moe_form(s, t).workspace_bytes);
  *workspace_bytes = most;
  return ok();
}

ccl_status ccl_moe_decode(const ccl_moe* moe, int64_t tokens, const void* x, int64_t x_ld, const float* logits,
                          int64_t logits_ld, const void* gate_up, const float* gate_up_scale, const void* down,
                          const float* down_scale, void* y, int64_t y_ld, int32_t* ids, float* probs,
                          void* workspace, int64_t workspace_bytes, void* stream) {
  ccl::MoeShape s;
  if (ccl_status st = check_moe(moe, tokens, &s)) return st;
  if (tokens == 0) return ok();
  if (!x || !logits || !gate_up || !down || !y) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  constexpr int64_t kMaxLd = (int64_t)1 << 22;    // 64 rows stay within 31-bit offsets
  if (x_ld < s.hidden || y_ld < s.hidden || logits_ld < s.experts || x_ld > kMaxLd || y_ld > kMaxLd || logits_ld > kMaxLd)
    return fail(CCL_ERR_INVALID_ARG, "a leading dimension is smaller than its row, or above 2^22");
  if (!aligned16(x) || x_ld % 8 || !aligned16(gate_up) || !aligned16(down))
    return fail(CCL_ERR_MISALIGNED_POINTER, "x (and its rows) and the weights must be 16-byte aligned");
  if (!aligned(logits, 4) || !aligned(gate_up_scale, 4) || !aligned(down_scale, 4) || !aligned(y, 2) ||
      !aligned(ids, 4) || !aligned(probs, 4))
    return fail(CCL_ERR_MISALIGNED_POINTER, "a pointer is not aligned to its elements");
  if (ccl_status st = check_workspace(ccl::moe_form(s, tokens).workspace_bytes, workspace, workspace_bytes)) return st;
  if (ccl_status st = check_device()) return st;
  ccl::MoeCall c;
  c.tokens = tokens;
  c.x = x;
  c.logits = logits;
  c.gate_up = gate_up;
  c.down = down;
  c.gate_up_scale = gate_up_scale;
  c.down_scale = down_scale;
  c.y = y;
  c.ids = ids;
  c.probs = probs;
  c.x_ld = x_ld;
  c.logits_ld = logits_ld;
  c.y_ld = y_ld;
  return hip_status(ccl::launch_moe(s, c, workspace, static_cast<hipStream_t>(stream)), "moe launch");
}

ccl_status ccl_orthogonalize_workspace(int64_t batch, int64_t rows, int64_t cols, int64_t* workspace_bytes) {
  if (!workspace_bytes) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  if (ccl_status s = check_ortho(batch, rows, cols)) return s;
  *workspace_bytes = batch && rows && cols ? ccl::ortho_form({batch, rows, cols}).workspace_bytes : 0;
  return ok();
}

ccl_status ccl_orthogonalize(int64_t batch, int64_t rows, int64_t cols, const void* G, ccl_dtype g_type, int64_t ld,
                             int64_t stride, int steps, const float* coeffs, float eps, void* O, int64_t o_ld,
                             int64_t o_stride, void* workspace, int64_t workspace_bytes, void* stream) {
  if (ccl_status s = check_ortho(batch, rows, cols)) return s;
  if (g_type != CCL_DT_BF16 && g_type != CCL_DT_FP32) return fail(CCL_ERR_INVALID_ARG, "G must be bf16 or fp32");
  if (steps < 0 || steps > 32) return fail(CCL_ERR_INVALID_ARG, "steps must be in 0..32");
  ccl::OrthoCall c;
  const float defaults[3] = {3.4445f, -4.7750f, 2.0315f};
  for (int i = 0; i < 3; ++i) {
    c.coeffs[i] = coeffs ? coeffs[i] : defaults[i];
    if (!std::isfinite(c.coeffs[i])) return fail(CCL_ERR_INVALID_ARG, "coefficients must be finite");
  }
  if (!std::isfinite(eps) || eps < 0.f) return fail(CCL_ERR_INVALID_ARG, "eps must be finite and not negative");
  if (batch == 0 || rows == 0 || cols == 0) return ok();
  if (!G || !O) return fail(CCL_ERR_INVALID_ARG, "NULL argument");
  constexpr int64_t kMaxStride = (int64_t)1 << 40;
  const int64_t span = (rows - 1) * std::max<int64_t>(ld, 0) + cols, o_span = (rows - 1) * std::max<int64_t>(o_ld, 0) + cols;
  if (ld < cols || o_ld < cols || ld > kMaxStride || o_ld > kMaxStride)
    return fail(CCL_ERR_INVALID_ARG, "a leading dimension is smaller than the row");
  if (batch > 1 && (stride < span || o_stride < o_span || stride > kMaxStride || o_stride > kMaxStride))
    return fail(CCL_ERR_INVALID_ARG, "matrices of the batch overlap");
  if (!aligned(G, g_type == CCL_DT_FP32 ? 4 : 2) || !aligned(O, 2))
    return fail(CCL_ERR_MISALIGNED_POINTER, "G and O must be aligned to their elements");
  const ccl::OrthoShape s{batch, rows, cols};
  if (ccl_status st = check_workspace(ccl::ortho_form(s).workspace_bytes, workspace, workspace_bytes)) return st;
  if (!aligned(workspace, 256)) return fail(CCL_ERR_MISALIGNED_POINTER, "the workspace must be 256-byte aligned");
  if (ccl_status st = check_device()) return st;
  c.G = G;
  c.f32 = g_type == CCL_DT_FP32;
  c.ld = ld;
  c.stride = batch > 1 ? stride : 0;
  c.O = O;
  c.o_ld = o_ld;
  c.o_stride = batch > 1 ? o_stride : 0;
  c.steps = steps;
  c.eps = eps;
  return hip_status(ccl::launch_orthogonalize(s, c, workspace, static_cast<hipStream_t>(stream)), "orthogonalize launch");
}

}  // extern "C"
