// Kernel launchers of the CCL library (device side lives in *.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../host/plan.hpp"

namespace ccl {

// Pack (row-major -> CCL) or unpack (CCL -> row-major) with ld.
hipError_t launch_copy(const Plan& p, int op, const void* rowmajor, int64_t ld, void* ccl_buf,
                       bool unpack, hipStream_t stream);
// Pack from a stored transpose (cols x rows, leading dimension ld).
hipError_t launch_pack_trans(const Plan& p, int op, const void* src, int64_t ld, void* dst,
                             hipStream_t stream);
// C = alpha A B + beta C with the given operand addressing; remap =
// XCD-aware tile map. C is read only when beta != 0. splits > 1 (remap
// only): split-K into the fp32 workspace ws, then a reduce launch.
// timeline (bf16, unsplit only): kTimelineWords uint64 per wave of every
// workgroup that has a tile, recorded by the kernel (debug launches).
hipError_t launch_gemm(const Plan& p, const void* A, const void* B, void* C,
                       const OperandAddr& a, const OperandAddr& b, const OperandAddr& c,
                       bool remap, float alpha, float beta, int splits, float* ws,
                       hipStream_t stream, uint64_t* timeline = nullptr);
constexpr int kTimelineWords = 8;
// The GEMM of form f with every tile's fp32 partials written to ws. md and
// wgm: the MFMA tile and the rows of the wave grid of the kernel that wrote
// them, which set their order.
hipError_t launch_gemm_partials(const Plan& p, const GemmForm& f, const void* A, const void* B,
                                const OperandAddr& a, const OperandAddr& b, float* ws, hipStream_t stream,
                                int* md, int* wgm);
// One ccl_gemm_fused (grad false) or ccl_gemm_fused_grad call. ws: the
// workspace of fused_form's size for the same arguments.
struct FusedCall {
  const void *A = nullptr, *B = nullptr;
  void* C = nullptr;               // C, or dZ
  const void* bias = nullptr;
  const void* R = nullptr;         // residual
  const void* Zin = nullptr;       // pre-activations read (grad)
  void* Zout = nullptr;            // pre-activations kept
  float* dbias = nullptr;          // column sums of dZ (grad)
  bool rowmajor = false, grad = false, gated = false, bias_f32 = false;
  int act = ACT_NONE;
  float alpha = 1.f, beta = 0.f;
  int64_t rows = 0;
};
hipError_t launch_gemm_fused(const Plan& p, const FusedCall& call, int splits, void* ws, hipStream_t stream);
// Split-K workspace for callers that cannot allocate device memory: a
// static device array of kScratchBytes in the library (one per GPU, held
// until the process ends). Returns its address on the current device,
// looked up once per device.
constexpr int64_t kScratchBytes = (int64_t)64 << 20;
hipError_t scratch_workspace(float** ws);
// Dispatch probe with an unsplit ccl_gemm's grid (4 int32 per workgroup).
hipError_t launch_dispatch_probe(const Plan& p, int32_t* out, hipStream_t stream);

// One ccl_moe_decode call; ws: moe_form's workspace.
struct MoeCall {
  int64_t tokens = 0;
  const void* x = nullptr;
  const float* logits = nullptr;
  const void* gate_up = nullptr;
  const void* down = nullptr;
  const float* gate_up_scale = nullptr;
  const float* down_scale = nullptr;
  void* y = nullptr;
  int32_t* ids = nullptr;
  float* probs = nullptr;
  int64_t x_ld = 0, logits_ld = 0, y_ld = 0;
};
hipError_t launch_moe(const MoeShape& s, const MoeCall& c, void* ws, hipStream_t stream);

// One ccl_orthogonalize call; ws: ortho_form's workspace.
struct OrthoCall {
  const void* G = nullptr;
  bool f32 = false;
  int64_t ld = 0, stride = 0;
  void* O = nullptr;
  int64_t o_ld = 0, o_stride = 0;
  int steps = 0;
  float coeffs[3] = {0.f, 0.f, 0.f};
  float eps = 0.f;
};
hipError_t launch_orthogonalize(const OrthoShape& s, const OrthoCall& c, void* ws, hipStream_t stream);

}  // namespace ccl
