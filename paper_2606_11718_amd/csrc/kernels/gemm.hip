// The GEMM kernels and their launches: the tile functions of gemm_tiles.hpp
// with the plain epilogue, the split-K reduce and the dispatch probe.
#include "gemm_tiles.hpp"

namespace ccl {

namespace {

template <int BM, int BN, int WGN>
__global__ void __launch_bounds__(128 * WGN, WGN / 2) gemm_kernel(GemmParams p) {
  // The host pass only needs the launch stub; the tile functions use
  // device-only buffer-resource builtins.
#if defined(__HIP_DEVICE_COMPILE__)
  k32_tile<BM, BN, WGN>(p);
#endif
}

template <int BM, int BN, bool RAGGED, bool BNT>
__global__ void __launch_bounds__(512, 2) gemm_k64_kernel(GemmParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  k64_tile<BM, BN, RAGGED, BNT, false>(p);
#endif
}

template <int BM, int BN, bool BNT>
__global__ void __launch_bounds__(512, 2) gemm_k64_far_kernel(GemmParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  k64_tile<BM, BN, false, BNT, true>(p);
#endif
}

__global__ void __launch_bounds__(512, 2) gemm_a2_kernel(GemmParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  a2_tile(p);
#endif
}

__global__ void __launch_bounds__(512, 2) gemm_fp8p_kernel(GemmParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  fp8p_tile(p);
#endif
}

template <int BM, int BN, int WGM, int WGN>
__global__ void __launch_bounds__(64 * WGM * WGN, WGM * WGN / 4) gemm_fp8s_kernel(GemmParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  fp8s_tile<BM, BN, WGM, WGN>(p);
#endif
}

// Records, per workgroup of the GEMM grid, the XCD it ran on and its tile.
__global__ void __launch_bounds__(64) dispatch_probe_kernel(TileMap map, int32_t tiles_m,
                                                            int32_t tiles_n, int32_t* out) {
  if (threadIdx.x != 0) return;
  uint32_t xcc;
  asm volatile("s_getreg_b32 %0, hwreg(HW_REG_XCC_ID)" : "=s"(xcc));
  int32_t pr, pc, ti, tj;
  int32_t* o = out + 4 * (int64_t)blockIdx.x;
  o[0] = (int32_t)(xcc & 0xf);
  if (map_tile(map, blockIdx.x, &pr, &pc, &ti, &tj)) {
    o[1] = pr * tiles_m + ti;
    o[2] = pc * tiles_n + tj;
    o[3] = pr * map.grid_c + pc;
  } else {
    o[1] = o[2] = o[3] = -1;
  }
}

}  // namespace

// Split-K workspace of ccl_gemm_splitk_noalloc: the fp32 partial tiles
// live in this array instead of caller memory. Each GPU holds its own copy
// (allocated when the library's code object is loaded on it). Nothing in it
// needs clearing: every K range writes its whole partial tile before the
// reduce launch reads it. Calls that overlap on one GPU share it and race.
static __device__ __align__(256) float scratch[kScratchBytes / sizeof(float)];

namespace {
constexpr int kScratchDevices = 64;
std::once_flag g_scratch_once[kScratchDevices];
float* g_scratch_ptr[kScratchDevices];
hipError_t g_scratch_err[kScratchDevices];
}  // namespace

// Host code must not pass `scratch` itself to a kernel (on the host the name
// is only a stand-in): the device address comes from the runtime, once per
// device, with that device current.
hipError_t scratch_workspace(float** ws) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kScratchDevices) return hipErrorInvalidDevice;
  std::call_once(g_scratch_once[dev], [dev] {
    void* ptr = nullptr;
    g_scratch_err[dev] = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
    g_scratch_ptr[dev] = static_cast<float*>(ptr);
  });
  if (g_scratch_err[dev] != hipSuccess) return g_scratch_err[dev];
  if (g_scratch_ptr[dev] == nullptr) return hipErrorInvalidSymbol;
  *ws = g_scratch_ptr[dev];
  return hipSuccess;
}

// Second launch of a split-K GEMM: sum the partials of every tile into C.
// md, waves and wgm are the MFMA tile, the waves and the rows of the wave grid
// of the kernel that wrote them, which set their fragment order.
static hipError_t launch_splitk_reduce(const Plan& p, GemmParams gp, int md, int waves,
                                       hipStream_t stream, int wgm = 2) {
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  gp.map = tile_map(p, 1);
  const dim3 grid((unsigned)splitk_reduce_workgroups(p));
  const GemmConfig& g = p.gemm;
#define CCL_REDUCE(BM_, BN_, WGN_, MD_) \
  hipLaunchKernelGGL((splitk_reduce_kernel<BM_, BN_, WGN_, MD_>), grid, dim3(256), 0, stream, gp)
#define CCL_REDUCE_MD(BM_, BN_, WGN_) \
  do { if (md == 16) CCL_REDUCE(BM_, BN_, WGN_, 16); else CCL_REDUCE(BM_, BN_, WGN_, 32); } while (0)
  if (g.tile_m == 256 && g.tile_n == 256 && waves == 8) CCL_REDUCE_MD(256, 256, 4);
  else if (g.tile_m == 256 && g.tile_n == 128 && waves == 8 && wgm == 4)
    hipLaunchKernelGGL((splitk_reduce_kernel<256, 128, 2, 16, 4>), grid, dim3(256), 0, stream, gp);
  else if (g.tile_m == 256 && g.tile_n == 128 && waves == 8) CCL_REDUCE(256, 128, 4, 16);
  else if (g.tile_m == 128 && g.tile_n == 256 && waves == 8) CCL_REDUCE(128, 256, 4, 16);
  else if (g.tile_m == 128 && g.tile_n == 128 && waves == 8) CCL_REDUCE(128, 128, 4, 16);
  else if (g.tile_m == 256 && g.tile_n == 256) CCL_REDUCE_MD(256, 256, 2);
  else if (g.tile_m == 256 && g.tile_n == 128) CCL_REDUCE_MD(256, 128, 2);
  else if (g.tile_m == 128 && g.tile_n == 256) CCL_REDUCE_MD(128, 256, 2);
  else if (g.tile_m == 128 && g.tile_n == 128) CCL_REDUCE_MD(128, 128, 2);
  else return hipErrorInvalidValue;
#undef CCL_REDUCE_MD
#undef CCL_REDUCE
  return hipGetLastError();
}

// The launch of form f's kernel. On return md and wgm are its MFMA tile and
// the rows of its wave grid, for the reduce of its partials.
static hipError_t launch_form(const GemmForm& f, const GemmParams& gp, hipStream_t stream, int* md_out,
                              int* wgm_out) {
  const dim3 grid((unsigned)f.workgroups);
  // MFMA tile and rows of the wave grid, for the reduce of split-K partials
  int &md = *md_out, &wgm = *wgm_out;
  md = 16;
  wgm = 2;
  const auto tile = [&](int m, int n) { return f.tile_m == m && f.tile_n == n; };
  switch (f.kernel) {
    case GemmKernel::FP8P:
      hipLaunchKernelGGL(gemm_fp8p_kernel, grid, dim3(TileFp8P::THREADS), 0, stream, gp);
      break;
    case GemmKernel::FP8X:
      hipLaunchKernelGGL((gemm_fp8x_kernel<256, 256, 4>), grid, dim3(Tile8x<256, 256, 4>::THREADS), 0,
                         stream, gp);
      break;
    case GemmKernel::FP8S:
#define CCL_LAUNCH8S(BM_, BN_, WGM_, WGN_)                                                  \
  hipLaunchKernelGGL((gemm_fp8s_kernel<BM_, BN_, WGM_, WGN_>), grid,                        \
                     dim3(Tile8s<BM_, BN_, WGM_, WGN_>::THREADS), 0, stream, gp)
      // wave tiles of 64x64 for 256x128 (a 4 x 2 grid reads 176 KiB of LDS per
      // stage, 2 x 4 208 KiB: 1.5-3.5 % faster), 64x64 and 64x32 otherwise
      wgm = f.tile_m == 256 ? 4 : 2;
      if (tile(256, 128)) CCL_LAUNCH8S(256, 128, 4, 2);
      else if (tile(128, 256)) CCL_LAUNCH8S(128, 256, 2, 4);
      else if (tile(128, 128)) CCL_LAUNCH8S(128, 128, 2, 4);
      else return hipErrorInvalidValue;
#undef CCL_LAUNCH8S
      break;
    case GemmKernel::FP8:
#define CCL_LAUNCH8(BM_, BN_, WGN_)                                                    \
  hipLaunchKernelGGL((gemm_fp8_kernel<BM_, BN_, WGN_>), grid, dim3(Tile8<BM_, BN_, WGN_>::THREADS), \
                     0, stream, gp)
      md = 32;
      if (tile(256, 256) && f.waves == 8) CCL_LAUNCH8(256, 256, 4);
      else if (tile(256, 256)) CCL_LAUNCH8(256, 256, 2);
      else if (tile(256, 128)) CCL_LAUNCH8(256, 128, 2);
      else if (tile(128, 256)) CCL_LAUNCH8(128, 256, 2);
      else if (tile(128, 128)) CCL_LAUNCH8(128, 128, 2);
      else return hipErrorInvalidValue;
#undef CCL_LAUNCH8
      break;
    case GemmKernel::K64:
#define CCL_LAUNCH64_AS(BM_, BN_, RAGGED_, BNT_)                                                   \
  hipLaunchKernelGGL((gemm_k64_kernel<BM_, BN_, RAGGED_, BNT_>), grid,                             \
                     dim3(Tile64<BM_, BN_>::THREADS), 0, stream, gp)
#define CCL_LAUNCH64(BM_, BN_)                                            \
  do {                                                                    \
    if (!f.ragged && f.stream_b) CCL_LAUNCH64_AS(BM_, BN_, false, true);  \
    else if (!f.ragged) CCL_LAUNCH64_AS(BM_, BN_, false, false);          \
    else if (f.stream_b) CCL_LAUNCH64_AS(BM_, BN_, true, true);           \
    else CCL_LAUNCH64_AS(BM_, BN_, true, false);                          \
  } while (0)
#define CCL_LAUNCH64_FAR(BM_, BN_)                                                                 \
  do {                                                                                             \
    if (f.stream_b)                                                                                \
      hipLaunchKernelGGL((gemm_k64_far_kernel<BM_, BN_, true>), grid, dim3(Tile64<BM_, BN_>::THREADS), 0, stream, gp);  \
    else                                                                                           \
      hipLaunchKernelGGL((gemm_k64_far_kernel<BM_, BN_, false>), grid, dim3(Tile64<BM_, BN_>::THREADS), 0, stream, gp); \
  } while (0)
      if (f.far && tile(256, 128)) CCL_LAUNCH64_FAR(256, 128);
      else if (f.far && tile(128, 256)) CCL_LAUNCH64_FAR(128, 256);
      else if (f.far && tile(128, 128)) CCL_LAUNCH64_FAR(128, 128);
      else if (f.far) return hipErrorInvalidValue;
      else if (tile(128, 192)) CCL_LAUNCH64(128, 192);
      else if (tile(128, 320)) CCL_LAUNCH64(128, 320);
      else if (tile(256, 128)) CCL_LAUNCH64(256, 128);
      else if (tile(128, 256)) CCL_LAUNCH64(128, 256);
      else if (tile(128, 128)) CCL_LAUNCH64(128, 128);
      else return hipErrorInvalidValue;
#undef CCL_LAUNCH64
#undef CCL_LAUNCH64_AS
#undef CCL_LAUNCH64_FAR
      break;
    case GemmKernel::A2:
      hipLaunchKernelGGL(gemm_a2_kernel, grid, dim3(TileA2::THREADS), 0, stream, gp);
      break;
    case GemmKernel::K32:
#define CCL_LAUNCH(BM_, BN_, WGN_)                                                     \
  hipLaunchKernelGGL((gemm_kernel<BM_, BN_, WGN_>), grid, dim3(Tile<BM_, BN_, WGN_>::THREADS), 0, \
                     stream, gp)
      if (tile(256, 256) && f.waves == 8) CCL_LAUNCH(256, 256, 4);
      else if (tile(256, 128) && f.waves == 8) CCL_LAUNCH(256, 128, 4);
      else if (tile(128, 256) && f.waves == 8) CCL_LAUNCH(128, 256, 4);
      else if (tile(128, 128) && f.waves == 8) CCL_LAUNCH(128, 128, 4);
      else if (tile(256, 256)) CCL_LAUNCH(256, 256, 2);
      else if (tile(256, 128)) CCL_LAUNCH(256, 128, 2);
      else if (tile(128, 256)) CCL_LAUNCH(128, 256, 2);
      else if (tile(128, 128)) CCL_LAUNCH(128, 128, 2);
      else return hipErrorInvalidValue;
#undef CCL_LAUNCH
      break;
  }
  return hipGetLastError();
}

hipError_t launch_gemm(const Plan& p, const void* A, const void* B, void* C,
                       const OperandAddr& a, const OperandAddr& b, const OperandAddr& c,
                       bool remap, float alpha, float beta, int splits, float* ws,
                       hipStream_t stream, uint64_t* timeline) {
  if (splits < 1 || (splits > 1 && (!remap || !ws))) return hipErrorInvalidValue;
  const GemmForm f = gemm_form(p, a, b, remap, splits, beta != 0.f);
  if (timeline && (p.ab_type != DT_BF16 || f.splits > 1)) return hipErrorInvalidValue;   // bf16 kernels only
  GemmParams gp;
  gemm_params(p, f, A, B, C, a, b, c, remap, &gp);
  gp.timeline = timeline;
  gp.ws = f.splits > 1 ? ws : nullptr;
  gp.alpha = alpha;
  gp.beta = beta;
  gp.epi = beta != 0.f ? 2 : (alpha != 1.f ? 1 : 0);
  int md, wgm;
  const hipError_t e = launch_form(f, gp, stream, &md, &wgm);
  if (e != hipSuccess || f.splits == 1) return e;
  return launch_splitk_reduce(p, gp, md, f.waves, stream, wgm);
}

hipError_t launch_gemm_partials(const Plan& p, const GemmForm& f, const void* A, const void* B,
                                const OperandAddr& a, const OperandAddr& b, float* ws, hipStream_t stream,
                                int* md, int* wgm) {
  GemmParams gp;
  gemm_params(p, f, A, B, nullptr, a, b, OperandAddr{0, 0, 0, 0}, true, &gp);
  gp.ws = ws;
  return launch_form(f, gp, stream, md, wgm);
}

hipError_t launch_dispatch_probe(const Plan& p, int32_t* out, hipStream_t stream) {
  OperandAddr a, b, c;
  ccl_addressing(p, &a, &b, &c);
  const GemmForm f = gemm_form(p, a, b, true, 1);
  hipLaunchKernelGGL(dispatch_probe_kernel, dim3((unsigned)f.workgroups), dim3(64), 0, stream, f.map,
                     f.map.tiles_m, f.map.tiles_n, out);
  return hipGetLastError();
}

}  // namespace ccl
