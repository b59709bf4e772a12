// ccl_gemm_fused and ccl_gemm_fused_grad: the GEMM's tile functions with the
// fused epilogues, the reduce that applies them to fp32 partials, and their
// launches.
#include "gemm_tiles.hpp"

namespace ccl {

namespace {

// The GEMM's tiles with the epilogue behind the K loop.
// WGN: columns of the wave grid, 4 or 2. A gated product on 192 or 320 columns
// takes 2, so that a wave's 16-column tiles are whole pairs of gate and up.
template <int BM, int BN, bool RAGGED, bool BNT, bool GRAD, int WGN = 4>
__global__ void __launch_bounds__(512, 2) fused_k64_kernel(FusedTileParams<GRAD> p) {
#if defined(__HIP_DEVICE_COMPILE__)
  k64_tile<BM, BN, RAGGED, BNT, false, WGN>(p);
#endif
}

template <int BM, int BN, bool GRAD>
__global__ void __launch_bounds__(512, 2) fused_k32_kernel(FusedTileParams<GRAD> p) {
#if defined(__HIP_DEVICE_COMPILE__)
  k32_tile<BM, BN, 4>(p);
#endif
}

template <bool GRAD>
__global__ void __launch_bounds__(512, 2) fused_a2_kernel(FusedTileParams<GRAD> p) {
#if defined(__HIP_DEVICE_COMPILE__)
  a2_tile(p);
#endif
}

template <bool GRAD>
__global__ void __launch_bounds__(512, 2) fused_fp8p_kernel(FusedTileParams<GRAD> p) {
#if defined(__HIP_DEVICE_COMPILE__)
  fp8p_tile(p);
#endif
}

template <int BM, int BN, int WGM, int WGN, bool GRAD>
__global__ void __launch_bounds__(64 * WGM * WGN, WGM * WGN / 4) fused_fp8s_kernel(FusedTileParams<GRAD> p) {
#if defined(__HIP_DEVICE_COMPILE__)
  fp8s_tile<BM, BN, WGM, WGN>(p);
#endif
}

// The simple form: the product's fp32 partial tiles (split-K ranges, or one
// range of the whole K) are read back from the workspace and summed in
// ascending range order, one float4 per thread, as splitk_reduce_kernel does.
// Bound by reading the partials; used for split-K and for the plans whose
// GEMM kernel has no fused epilogue of its own.
template <int BM, int BN, int WGN, int MD, int WGM, bool GRAD>
__global__ void __launch_bounds__(256) fused_reduce_kernel(FusedParams p) {
  using L = AccLayout<MD>;
  constexpr int WM = BM / WGM, WN = BN / WGN;
  constexpr int TM = WM / MD, TN = WN / MD;
  constexpr int kChunks = BM * BN / (4 * 256);
  const int64_t slot = blockIdx.x >> 3;
  const int32_t chunk = (int32_t)(slot % kChunks);
  int32_t pr, pc, ti, tj, split;
  if (!map_tile(p.map, ((slot / kChunks) << 3) | (blockIdx.x & 7), &pr, &pc, &ti, &tj, &split)) return;
  const int32_t f = chunk * 256 + threadIdx.x;
  const int lane = f & 63;
  int r = f >> 6;
  const int q = r % L::Q;
  r /= L::Q;
  const int nt = r % TN;
  r /= TN;
  const int mt = r % TM;
  const int wave = r / TM;
  const int wm = wave / (BN / WN), wn = wave % (BN / WN);
  const int64_t m = ti * BM + wm * WM + mt * MD + L::row(lane);   // row in the partition
  const int n = tj * BN + wn * WN + nt * MD + L::col(lane, q);    // column of D in the partition
  const FusedEpi& e = p.e;
  const bool live = pr * e.part_rows + m < e.rows;
  const int32_t S = p.splits_total;
  const float4* part = reinterpret_cast<const float4*>(p.ws + tile_id(p, pr, pc, ti, tj) * S * (BM * BN));
  auto sum = [&](int32_t at) {
    f32x4 o{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < S; ++s) o += *reinterpret_cast<const f32x4*>(part + at + (int64_t)s * (BM * BN / 4));
    return o * p.alpha;
  };
  const int64_t c_at = pr * p.c.part + pc * p.c.slice + m * p.c.ld;
  const int64_t z_at = pr * e.z.part + pc * e.z.slice + m * e.z.ld;
  auto put = [](uint16_t* base, int64_t at, f32x4 v) { *reinterpret_cast<uint2*>(base + at) = f32_to_bf16x4(v); };
  uint16_t* C = static_cast<uint16_t*>(p.C);
  const f32x4 zero{0.f, 0.f, 0.f, 0.f};
  if constexpr (!GRAD) {
    // The up columns' threads leave: the gate columns' threads read both. The
    // up's float4 lies in the next MFMA tile (16 wide) or two groups on (32).
    constexpr int kUp = MD == 16 ? 64 * L::Q : 2 * 64;
    if (e.gated && (n & 16)) return;
    f32x4 z = live ? sum(f) + bias4(e, pc * (int64_t)e.part_cols + n) : zero;
    f32x4 u = e.gated && live ? sum(f + kUp) + bias4(e, pc * (int64_t)e.part_cols + n + 16) : zero;
    if (e.Zout) {
      put(e.Zout, z_at + n, z);
      if (e.gated) put(e.Zout, z_at + n + 16, u);
    }
    f32x4 o;
    const ActCoef k = act_coef(e.act);
    with_act(e.act, [&](auto cls) {
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = act_value<decltype(cls)::value>(k, z[j]);
    });
    if (e.gated) o *= u;
    const int cn = e.gated ? ((n >> 5) << 4) | (n & 15) : n;
    if (!live) {
      o = zero;
    } else if (e.R) {
      const f32x4 res = bf16x4_to_f32(*reinterpret_cast<const uint2*>(e.R + c_at + cn));
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = __builtin_fmaf(e.beta, res[j], o[j]);
    }
    put(C, c_at + cn, o);
  } else {
    const int zn = e.gated ? wide_col(n) : n;
    f32x4 g = zero, u = zero;
    if (live) {
      const f32x4 d = sum(f);
      const f32x4 z = e.Zin ? bf16x4_to_f32(*reinterpret_cast<const uint2*>(e.Zin + z_at + zn)) : zero;
      const f32x4 zu = e.gated ? bf16x4_to_f32(*reinterpret_cast<const uint2*>(e.Zin + z_at + zn + 16)) : zero;
      const ActCoef k = act_coef(e.act);
      with_act(e.act, [&](auto cls) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float grad;
          const float value = act_value_grad<decltype(cls)::value>(k, z[j], &grad);
          g[j] = d[j] * grad;
          if (e.gated) {
            g[j] *= zu[j];
            u[j] = d[j] * value;
          }
        }
      });
    }
    put(C, c_at + zn, g);
    if (e.gated) put(C, c_at + zn + 16, u);
    if (e.colsum) {
      // The MD lanes of a column group hold MD rows of four columns.
      const int64_t block = (pr * e.part_rows + m) / MD;
      float* to = e.colsum + block * e.z_cols + (e.gated ? 2 : 1) * pc * (int64_t)e.part_cols + zn;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (half && !e.gated) break;
        f32x4 v = half ? u : g;
#pragma unroll
        for (int x = 1; x < MD; x <<= 1)
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] += __shfl_xor(v[j], x);
        if ((lane & (MD - 1)) == 0) *reinterpret_cast<f32x4*>(to + 16 * half) = v;
      }
    }
  }
}

// Column sums over the row blocks, in a fixed order: thread (g, c) adds the
// blocks g, g + 4, ... of its column, then the four are added.
__global__ void __launch_bounds__(256) bias_reduce_kernel(const float* part, int64_t blocks, int64_t cols, float* out) {
  __shared__ float sm[4][64];
  const int c = threadIdx.x & 63, g = threadIdx.x >> 6;
  const int64_t col = (int64_t)blockIdx.x * 64 + c;
  float v = 0.f;
  if (col < cols) {
#pragma unroll 8
    for (int64_t b = g; b < blocks; b += 4) v += part[b * cols + col];
  }
  sm[g][c] = v;
  __syncthreads();
  if (g == 0 && col < cols) out[col] = ((sm[0][c] + sm[1][c]) + sm[2][c]) + sm[3][c];
}

}  // namespace

// The workspace form of the fused epilogue: partials, then the reduce.
template <bool GRAD>
static hipError_t launch_fused_reduce(const Plan& p, FusedParams fp, int md, int waves, int wgm,
                                      hipStream_t stream) {
  fp.map = tile_map(p, 1);
  const dim3 grid((unsigned)splitk_reduce_workgroups(p));
  const GemmConfig& g = p.gemm;
  const auto tile = [&](int m, int n) { return g.tile_m == m && g.tile_n == n; };
#define CCL_FUSED_REDUCE(BM_, BN_, WGN_, MD_, WGM_) \
  hipLaunchKernelGGL((fused_reduce_kernel<BM_, BN_, WGN_, MD_, WGM_, GRAD>), grid, dim3(256), 0, stream, fp)
  if (waves == 8 && md == 16) {
    if (tile(256, 256)) CCL_FUSED_REDUCE(256, 256, 4, 16, 2);
    else if (tile(256, 128) && wgm == 4) CCL_FUSED_REDUCE(256, 128, 2, 16, 4);
    else if (tile(256, 128)) CCL_FUSED_REDUCE(256, 128, 4, 16, 2);
    else if (tile(128, 256)) CCL_FUSED_REDUCE(128, 256, 4, 16, 2);
    else if (tile(128, 128)) CCL_FUSED_REDUCE(128, 128, 4, 16, 2);
    else return hipErrorInvalidValue;
  } else if (waves == 8) {
    if (tile(256, 256)) CCL_FUSED_REDUCE(256, 256, 4, 32, 2);
    else return hipErrorInvalidValue;
  } else if (md == 16) {
    if (tile(256, 256)) CCL_FUSED_REDUCE(256, 256, 2, 16, 2);
    else if (tile(256, 128)) CCL_FUSED_REDUCE(256, 128, 2, 16, 2);
    else if (tile(128, 256)) CCL_FUSED_REDUCE(128, 256, 2, 16, 2);
    else if (tile(128, 128)) CCL_FUSED_REDUCE(128, 128, 2, 16, 2);
    else return hipErrorInvalidValue;
  } else {
    if (tile(256, 256)) CCL_FUSED_REDUCE(256, 256, 2, 32, 2);
    else if (tile(256, 128)) CCL_FUSED_REDUCE(256, 128, 2, 32, 2);
    else if (tile(128, 256)) CCL_FUSED_REDUCE(128, 256, 2, 32, 2);
    else if (tile(128, 128)) CCL_FUSED_REDUCE(128, 128, 2, 32, 2);
    else return hipErrorInvalidValue;
  }
#undef CCL_FUSED_REDUCE
  return hipGetLastError();
}

// A gated product on 128 x 192 or 128 x 320 tiles.
template <int BM, int BN>
static void launch_pairs(const GemmForm& f, const FusedParams& fp, hipStream_t stream) {
  FusedTileParams<false> p;
  static_cast<FusedParams&>(p) = fp;
  const dim3 grid((unsigned)f.workgroups), block(512);
#define CCL_PAIRS(R_, B_) hipLaunchKernelGGL((fused_k64_kernel<BM, BN, R_, B_, false, 2>), grid, block, 0, stream, p)
  if (!f.ragged && f.stream_b) CCL_PAIRS(false, true);
  else if (!f.ragged) CCL_PAIRS(false, false);
  else if (f.stream_b) CCL_PAIRS(true, true);
  else CCL_PAIRS(true, false);
#undef CCL_PAIRS
}

// A form with kernels of its own here (FusedForm::own): with the epilogue, or,
// with a workspace, the partials of the tiles that have valid rows.
template <bool GRAD>
static hipError_t launch_own(const GemmForm& f, const FusedParams& fp, hipStream_t stream) {
  FusedTileParams<GRAD> p;
  static_cast<FusedParams&>(p) = fp;
  const dim3 grid((unsigned)f.workgroups), block(512);
  const auto tile = [&](int m, int n) { return f.tile_m == m && f.tile_n == n; };
#define CCL_FUSED(...) hipLaunchKernelGGL((__VA_ARGS__), grid, block, 0, stream, p)
#define CCL_FUSED_K64(BM_, BN_, WGN_)                                                            \
  do {                                                                                           \
    if (!f.ragged && f.stream_b) CCL_FUSED(fused_k64_kernel<BM_, BN_, false, true, GRAD, WGN_>); \
    else if (!f.ragged) CCL_FUSED(fused_k64_kernel<BM_, BN_, false, false, GRAD, WGN_>);         \
    else if (f.stream_b) CCL_FUSED(fused_k64_kernel<BM_, BN_, true, true, GRAD, WGN_>);          \
    else CCL_FUSED(fused_k64_kernel<BM_, BN_, true, false, GRAD, WGN_>);                         \
  } while (0)
  const bool pairs = !GRAD && fp.e.gated;
  if (f.kernel == GemmKernel::A2) CCL_FUSED(fused_a2_kernel<GRAD>);
  else if (f.kernel == GemmKernel::FP8P) CCL_FUSED(fused_fp8p_kernel<GRAD>);
  else if (f.kernel == GemmKernel::K64 && tile(256, 128)) CCL_FUSED_K64(256, 128, 4);
  else if (f.kernel == GemmKernel::K64 && tile(128, 256)) CCL_FUSED_K64(128, 256, 4);
  else if (f.kernel == GemmKernel::K64 && tile(128, 128)) CCL_FUSED_K64(128, 128, 4);
  else if (f.kernel == GemmKernel::K64 && tile(128, 192) && !pairs) CCL_FUSED_K64(128, 192, 4);
  else if (f.kernel == GemmKernel::K64 && tile(128, 320) && !pairs) CCL_FUSED_K64(128, 320, 4);
  else if (f.kernel == GemmKernel::K64 && tile(128, 192)) launch_pairs<128, 192>(f, fp, stream);
  else if (f.kernel == GemmKernel::K64 && tile(128, 320)) launch_pairs<128, 320>(f, fp, stream);
  else if (f.kernel == GemmKernel::K32 && tile(256, 256)) CCL_FUSED(fused_k32_kernel<256, 256, GRAD>);
  else if (f.kernel == GemmKernel::K32 && tile(256, 128)) CCL_FUSED(fused_k32_kernel<256, 128, GRAD>);
  else if (f.kernel == GemmKernel::K32 && tile(128, 256)) CCL_FUSED(fused_k32_kernel<128, 256, GRAD>);
  else if (f.kernel == GemmKernel::K32 && tile(128, 128)) CCL_FUSED(fused_k32_kernel<128, 128, GRAD>);
  else if (f.kernel == GemmKernel::FP8S && tile(256, 128)) CCL_FUSED(fused_fp8s_kernel<256, 128, 4, 2, GRAD>);
  else if (f.kernel == GemmKernel::FP8S && tile(128, 256)) CCL_FUSED(fused_fp8s_kernel<128, 256, 2, 4, GRAD>);
  else if (f.kernel == GemmKernel::FP8S && tile(128, 128)) CCL_FUSED(fused_fp8s_kernel<128, 128, 2, 4, GRAD>);
  else return hipErrorInvalidValue;
#undef CCL_FUSED_K64
#undef CCL_FUSED
  return hipGetLastError();
}

hipError_t launch_gemm_fused(const Plan& plan, const FusedCall& call, int splits, void* ws, hipStream_t stream) {
  const int wide = call.gated ? 2 : 1;        // matrices of half or twice D's columns
  const int moved = call.grad ? (call.Zin ? 4 : 2) * wide : (call.R ? 4 : 2) / wide + (call.Zout ? 2 : 0);
  const FusedForm ff = fused_form(plan, call.rowmajor, splits, call.grad, call.gated, call.dbias != nullptr,
                                  call.rows, moved);
  const GemmForm& f = ff.gemm;
  Plan p = plan;
  p.gemm = ff.config;
  p.gemm.wide_n = 0;
  FusedParams fp;
  gemm_params(p, f, call.A, call.B, call.C, ff.a, ff.b, ff.c, ff.remap, &fp);
  fp.live = ff.live;
  fp.alpha = call.alpha;
  fp.c_nt = ff.c_nt ? 1 : 0;
  fp.e.bias = call.bias;
  fp.e.R = static_cast<const uint16_t*>(call.R);
  fp.e.Zin = static_cast<const uint16_t*>(call.Zin);
  fp.e.Zout = static_cast<uint16_t*>(call.Zout);
  fp.e.colsum = call.dbias ? reinterpret_cast<float*>(static_cast<char*>(ws) + ff.partial_bytes) : nullptr;
  fp.e.z = ff.z;
  fp.e.rows = call.rows;
  fp.e.part_rows = p.part_rows();
  fp.e.z_cols = ff.z_cols;
  fp.e.part_cols = (int32_t)p.part_cols();
  fp.e.act = call.act;
  fp.e.gated = call.gated ? 1 : 0;
  fp.e.bias_f32 = call.bias_f32 ? 1 : 0;
  fp.e.beta = call.beta;
  hipError_t e;
  if (!ff.direct) fp.ws = static_cast<float*>(ws);
  if (ff.own) e = call.grad ? launch_own<true>(f, fp, stream) : launch_own<false>(f, fp, stream);
  if (ff.direct) {
    if (e != hipSuccess) return e;
  } else {
    int md = 16, wgm = f.kernel == GemmKernel::FP8S && f.tile_m == 256 ? 4 : 2;
    if (!ff.own) e = launch_gemm_partials(p, f, call.A, call.B, ff.a, ff.b, fp.ws, stream, &md, &wgm);
    if (e != hipSuccess) return e;
    e = call.grad ? launch_fused_reduce<true>(p, fp, md, f.waves, wgm, stream)
                  : launch_fused_reduce<false>(p, fp, md, f.waves, wgm, stream);
  }
  if (e != hipSuccess || !call.dbias) return e;
  hipLaunchKernelGGL(bias_reduce_kernel, dim3((unsigned)((ff.z_cols + 63) / 64)), dim3(256), 0, stream, fp.e.colsum,
                     (call.rows + ff.sum_rows - 1) / ff.sum_rows, ff.z_cols, call.dbias);
  return hipGetLastError();
}


}  // namespace ccl
