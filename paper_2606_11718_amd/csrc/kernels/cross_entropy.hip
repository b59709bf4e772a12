// Softmax cross entropy of z = scale X W^T (tokens x vocabulary) against target
// tokens, and its gradients (ccl_cross_entropy, ccl_cross_entropy_grad):
//   lse = log sum_v exp(z_v),  loss = lse - z_t,  p = exp(z - lse)
//   dX = P' W,  dW = P'^T X,  P'_v = g scale (p_v - [v = t])
// for a block of tokens at a time:
//   logits   tiles of X W^T that stay in registers: each leaves the maximum m
//            and sum of exp(z - m) of every row (fp32), the target's z, and for
//            the gradient e = exp(z - m) in bf16
//   combine  rows' lse and loss from the tiles' m and sums, in tile order
//   scale    e -> P', in place: e exp(m - lse) g scale; the target's p - 1 is
//            expm1(z_t - lse) of the fp32 z_t, since from a rounded p it would
//            lose everything where p is near 1
//   dX, dW   products of P' with W and X
// Logits in fp32 exist nowhere in memory; P' is kept for a block, 2 bytes each,
// so that neither gradient has to recompute them (6 T D V operations rather
// than 8). Rounded to bf16: e, P' (2^-8 each at most), dX and dW once.
#include "product.hpp"

#include "train_kernels.hpp"

namespace ccl {

namespace {

struct LogitsParams {
  const uint16_t *X, *W;
  const int64_t* targets;
  float* target_z;         // [tokens]
  float2* stat;            // [tokens][tiles_n]: maximum, sum
  uint16_t* E;             // [tokens][e_ld], or null
  int64_t x_ld, w_ld, e_ld;
  int32_t tokens, vocab, hidden, e_cols;
  int32_t tiles_m, tiles_n, group, chunk;
  float scale;
};

// Tile `id` in a raster of `group` tile rows, column by column.
__device__ __forceinline__ void raster(int64_t id, int32_t tiles_m, int32_t tiles_n, int32_t group, int32_t* ti, int32_t* tj) {
  const int32_t per = group * tiles_n, r = (int32_t)(id / per), first = r * group, h = min(group, tiles_m - first);
  const int32_t w = (int32_t)(id - (int64_t)r * per);
  *tj = __builtin_amdgcn_readfirstlane(w / h);
  *ti = __builtin_amdgcn_readfirstlane(first + w - w / h * h);
}

template <int BM, int BN, int NS, int WGN>
__global__ void __launch_bounds__(512, NS * (BM + BN) * 128 <= 80 * 1024 ? 4 : 2) logits_kernel(LogitsParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  using T = ProductTile<BM, BN, true, true, NS, WGN>;
  __shared__ __attribute__((aligned(1024))) char sm[T::LDS];
  const int64_t id = dealt_tile(p.chunk);
  if (id >= (int64_t)p.tiles_m * p.tiles_n) return;
  int32_t ti, tj;
  raster(id, p.tiles_m, p.tiles_n, p.group, &ti, &tj);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wn = wave % WGN;
  const int32_t rows = min(BM, p.tokens - ti * BM), cols = min(BN, p.vocab - tj * BN);
  f32x4 acc[T::TM][T::TN];
  product<T>(Side{p.X + (int64_t)ti * BM * p.x_ld, p.x_ld, rows, p.hidden},
             Side{p.W + (int64_t)tj * BN * p.w_ld, p.w_ld, cols, p.hidden}, 0, (p.hidden + 63) / 64, acc, sm, tid,
             [](int r) { return r; });
  float* const part = reinterpret_cast<float*>(sm);     // [WGN][BM]
  float* const whole = part + WGN * BM;                 // [BM]: the tile's maxima
  // rows' maxima over a wave's columns, then over the waves
  float top[T::TM];
#pragma unroll
  for (int mt = 0; mt < T::TM; ++mt) top[mt] = -INFINITY;
  each4<T>(tid, [&](int mt, int nt, int r, int c) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      acc[mt][nt][j] = c + j < cols ? acc[mt][nt][j] * p.scale : -INFINITY;
      top[mt] = fmaxf(top[mt], acc[mt][nt][j]);
    }
  });
  const int r0 = (wave / WGN) * T::WM + (lane & 15);
#pragma unroll
  for (int mt = 0; mt < T::TM; ++mt) {
    top[mt] = fmaxf(top[mt], __shfl_xor(top[mt], 16));
    top[mt] = fmaxf(top[mt], __shfl_xor(top[mt], 32));
    if (lane < 16) part[wn * BM + r0 + 16 * mt] = top[mt];
  }
  __syncthreads();
  float sum[T::TM];
#pragma unroll
  for (int mt = 0; mt < T::TM; ++mt) {
#pragma unroll
    for (int w = 0; w < WGN; ++w) top[mt] = fmaxf(top[mt], part[w * BM + r0 + 16 * mt]);
    if (wn == 0 && lane < 16) whole[r0 + 16 * mt] = top[mt];
    sum[mt] = 0.f;
    // the target's logit
    const int32_t row = ti * BM + r0 + 16 * mt;
    if (row < p.tokens) {
      const int64_t t = p.targets[row] - (int64_t)tj * BN - wn * T::WN - 4 * (lane >> 4);
#pragma unroll
      for (int nt = 0; nt < T::TN; ++nt)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (t == 16 * nt + j && tj * BN + wn * T::WN + 4 * (lane >> 4) + 16 * nt + j < p.vocab) p.target_z[row] = acc[mt][nt][j];
    }
  }
  each4<T>(tid, [&](int mt, int nt, int r, int c) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      acc[mt][nt][j] = __builtin_amdgcn_exp2f((acc[mt][nt][j] - top[mt]) * kLog2e);
      sum[mt] += acc[mt][nt][j];
    }
  });
  __syncthreads();
#pragma unroll
  for (int mt = 0; mt < T::TM; ++mt) {
    sum[mt] += __shfl_xor(sum[mt], 16);
    sum[mt] += __shfl_xor(sum[mt], 32);
    if (lane < 16) part[wn * BM + r0 + 16 * mt] = sum[mt];
  }
  __syncthreads();
  if (tid < rows) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < WGN; ++w) s += part[w * BM + tid];
    p.stat[(int64_t)(ti * BM + tid) * p.tiles_n + tj] = make_float2(whole[tid], s);
  }
  if (!p.E) return;
  __syncthreads();
  const auto e = staged<BM, BN>(sm);
  each4<T>(tid, [&](int mt, int nt, int r, int c) __attribute__((always_inline)) { *e.at(r, c) = f32_to_bf16x4(acc[mt][nt]); });
  staged_barrier();
  // columns past the vocabulary up to e_cols: exp(-inf) = 0
  tile_out<BM, BN, 512>(e, p.E + (int64_t)ti * BM * p.e_ld, p.e_ld, rows, tid,
                        [&](int c) { return tj * BN + 8 * c < p.e_cols ? tj * BN + 8 * c : -1; });
#endif
}

struct CombineParams {
  const float2* stat;
  const float* target_z;
  const int64_t* targets;
  const float* dloss;      // [tokens] or null
  float *loss, *lse;       // or null
  float2* factor;          // [tokens]: lse; g scale, 0 for a token without a target
  const uint16_t* X;       // rows copied to `rows`, zeros where the factor is 0 (null: not needed)
  uint16_t* rows;
  int64_t x_ld;
  int32_t tokens, vocab, tiles_n, hidden;
  float scale, dloss_scale;
};

// One wave a token: the tiles' sums brought to their common maximum. For dW the
// tokens' x are copied without those that add nothing to it: 0 times whatever a
// padding row holds need not be 0.
__global__ void __launch_bounds__(256) combine_kernel(CombineParams p) {
  const int32_t row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (row >= p.tokens) return;
  const float2* s = p.stat + (int64_t)row * p.tiles_n;
  float top = -INFINITY;
  for (int i = lane; i < p.tiles_n; i += 64) top = fmaxf(top, s[i].x);
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
  float sum = 0.f;
  for (int i = lane; i < p.tiles_n; i += 64) sum += s[i].y * __builtin_amdgcn_exp2f((s[i].x - top) * kLog2e);
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x);
  const float lse = top + logf(sum);
  const int64_t t = p.targets[row];
  const bool live = t >= 0 && t < p.vocab;
  const float g = live ? (p.dloss ? p.dloss[row] : 1.f) * p.dloss_scale * p.scale : 0.f;
  if (p.rows) {
    const uint4* from = reinterpret_cast<const uint4*>(p.X + row * p.x_ld);
    uint4* to = reinterpret_cast<uint4*>(p.rows + (int64_t)row * p.hidden);
    for (int i = lane; i < p.hidden / 8; i += 64) to[i] = g != 0.f ? from[i] : make_uint4(0, 0, 0, 0);
  }
  if (lane) return;
  if (p.loss) p.loss[row] = live ? lse - p.target_z[row] : 0.f;
  if (p.lse) p.lse[row] = lse;
  if (p.factor) p.factor[row] = make_float2(lse, g);
}

struct ScaleParams {
  uint16_t* E;
  const float2 *stat, *factor;
  const float* target_z;
  const int64_t* targets;
  int64_t e_ld;
  int32_t vocab, e_cols, tiles_n, tile_shift;
};

// e -> P', eight a thread.
__global__ void __launch_bounds__(256) scale_kernel(ScaleParams p) {
  const int32_t row = blockIdx.y, col = (blockIdx.x * 256 + threadIdx.x) * 8;
  if (col >= p.e_cols) return;
  uint4* at = reinterpret_cast<uint4*>(p.E + row * p.e_ld + col);
  const float2 f = p.factor[row];
  if (f.y == 0.f) {        // no target, or a weight of 0: also where e is not a number
    *at = make_uint4(0, 0, 0, 0);
    return;
  }
  const uint4 e = *at;
  const float k = __builtin_amdgcn_exp2f((p.stat[(int64_t)row * p.tiles_n + (col >> p.tile_shift)].x - f.x) * kLog2e) * f.y;
  f32x4 lo = bf16x4_to_f32(make_uint2(e.x, e.y)) * k, hi = bf16x4_to_f32(make_uint2(e.z, e.w)) * k;
  const int64_t t = p.targets[row] - col;
  if (t >= 0 && t < 8) {
    const float v = expm1f(p.target_z[row] - f.x) * f.y;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (t == j) lo[j] = v;
      if (t == 4 + j) hi[j] = v;
    }
  }
  const uint2 a = f32_to_bf16x4(lo), b = f32_to_bf16x4(hi);
  *at = make_uint4(a.x, a.y, b.x, b.y);
}

// A plain product out = U V' (+ add) (+ out), or fp32 partial sums of K ranges.
struct PlainParams {
  const uint16_t *U, *V;
  int64_t ldu, ldv, ld_out;
  void* out;               // bf16, or fp32 with f32
  const float* add;        // m x n without gaps, or null
  float* part;             // [splits][m][n], or null
  int32_t m, n, ku, kv, ksteps;
  int32_t mu, nv;          // columns that U and V have (RC sides, whole 16 bytes)
  int32_t tiles_m, tiles_n, group, chunk, splits, ksplit;
  int32_t f32, accumulate;
};

template <int BM, int BN, int NS, int WGN, bool UK, bool VK>
__global__ void __launch_bounds__(512, NS * (BM + BN) * 128 <= 80 * 1024 ? 4 : 2) plain_kernel(PlainParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  using T = ProductTile<BM, BN, UK, VK, NS, WGN>;
  __shared__ __attribute__((aligned(1024))) char sm[T::LDS];
  int64_t id = dealt_tile(p.chunk);
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
  if (id >= tiles * p.splits) return;
  const int32_t split = __builtin_amdgcn_readfirstlane((int32_t)(id / tiles));
  id -= split * tiles;
  int32_t ti, tj;
  raster(id, p.tiles_m, p.tiles_n, p.group, &ti, &tj);
  const int tid = threadIdx.x;
  const int32_t s0 = split * p.ksplit, steps = min(p.ksplit, p.ksteps - s0);
  const int32_t m = min(BM, p.m - ti * BM), n = min(BN, p.n - tj * BN);
  const Side u = UK ? Side{p.U + (int64_t)ti * BM * p.ldu, p.ldu, m, p.ku}
                    : Side{p.U + ti * BM, p.ldu, min(BM, p.mu - ti * BM), p.ku};
  const Side v = VK ? Side{p.V + (int64_t)tj * BN * p.ldv, p.ldv, n, p.kv}
                    : Side{p.V + tj * BN, p.ldv, min(BN, p.nv - tj * BN), p.kv};
  // a range ends where the next begins
  const int32_t end = (s0 + steps) * 64;
  f32x4 acc[T::TM][T::TN];
  product<T>(Side{u.base, u.ld, u.extent, min(u.k, end)}, Side{v.base, v.ld, v.extent, min(v.k, end)}, s0 * 64, steps, acc,
             sm, tid, [](int r) { return r; });
  if (p.part) {
    float* const to = p.part + ((int64_t)split * p.m + ti * BM) * p.n + tj * BN;
    each4<T>(tid, [&](int mt, int nt, int r, int c) __attribute__((always_inline)) {
      if (r < m && c < n) *reinterpret_cast<f32x4*>(to + (int64_t)r * p.n + c) = acc[mt][nt];
    });
    return;
  }
  const int64_t corner = (int64_t)ti * BM * p.ld_out + tj * BN;
  const float* const add = p.add ? p.add + (int64_t)ti * BM * p.n + tj * BN : nullptr;
  if (p.f32) {
    float* const to = static_cast<float*>(p.out) + corner;
    each4<T>(tid, [&](int mt, int nt, int r, int c) __attribute__((always_inline)) {
      if (r >= m || c >= n) return;
      f32x4* at = reinterpret_cast<f32x4*>(to + r * p.ld_out + c);
      f32x4 o = acc[mt][nt];
      if (add) o += *reinterpret_cast<const f32x4*>(add + (int64_t)r * p.n + c);
      if (p.accumulate) o += *at;
      *at = o;
    });
    return;
  }
  uint16_t* const to = static_cast<uint16_t*>(p.out) + corner;
  const auto s = staged<BM, BN>(sm);
  each4<T>(tid, [&](int mt, int nt, int r, int c) __attribute__((always_inline)) {
    f32x4 o = acc[mt][nt];
    if (r < m && c < n) {
      if (add) o += *reinterpret_cast<const f32x4*>(add + (int64_t)r * p.n + c);
      if (p.accumulate) o += bf16x4_to_f32(*reinterpret_cast<const uint2*>(to + r * p.ld_out + c));
    }
    *s.at(r, c) = f32_to_bf16x4(o);
  });
  staged_barrier();
  tile_out<BM, BN, 512>(s, to, p.ld_out, m, tid, [&](int c) { return 8 * c < n ? 8 * c : -1; });
#endif
}

// The ranges' sums in order, rounded: four elements a thread.
__global__ void __launch_bounds__(256) ranges_kernel(const float* part, int32_t splits, int64_t elems, int32_t n, uint16_t* out,
                                                     int64_t ld) {
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (at >= elems) return;
  f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int32_t s = 0; s < splits; ++s) v += *reinterpret_cast<const f32x4*>(part + s * elems + at);
  const int64_t r = at / n, c = at - r * n;
  *reinterpret_cast<uint2*>(out + r * ld + c) = f32_to_bf16x4(v);
}

// dW without tokens.
__global__ void __launch_bounds__(256) zero_kernel(char* out, int64_t rows, int64_t row_chunks, int64_t ld_bytes) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= rows * row_chunks) return;
  const int64_t r = at / row_chunks;
  *reinterpret_cast<uint4*>(out + r * ld_bytes + (at - r * row_chunks) * 16) = make_uint4(0, 0, 0, 0);
}

template <bool UK, bool VK>
hipError_t launch_plain(const ProductForm& f, PlainParams p, hipStream_t stream) {
  p.tiles_m = f.tiles_m;
  p.tiles_n = f.tiles_n;
  p.group = f.group;
  p.chunk = f.chunk;
  p.splits = f.splits;
  p.ksplit = f.ksplit;
  const dim3 grid((unsigned)f.workgroups), block(512);
  if (f.tile_m == 64) hipLaunchKernelGGL((plain_kernel<64, 128, 2, 4, UK, VK>), grid, block, 0, stream, p);
  else if (f.tile_m == 256) hipLaunchKernelGGL((plain_kernel<256, 256, 2, 4, UK, VK>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((plain_kernel<128, 128, 2, 4, UK, VK>), grid, block, 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cross_entropy(const VocabShape& s, const VocabCall& c, void* ws, hipStream_t stream) {
  if (c.tokens == 0) {
    if (!c.grad || !c.dw || c.accumulate) return hipSuccess;
    const int64_t size = c.dw_f32 ? 4 : 2, chunks = s.hidden * size / 16;
    hipLaunchKernelGGL(zero_kernel, dim3((unsigned)((s.vocab * chunks + 255) / 256)), dim3(256), 0, stream,
                       static_cast<char*>(c.dw), s.vocab, chunks, c.dw_ld * size);
    return hipGetLastError();
  }
  const VocabForm f = vocab_form(s, c.tokens, c.grad);
  char* const at = static_cast<char*>(ws);
  float* const target_z = reinterpret_cast<float*>(at + f.target_at);
  float2* const factor = reinterpret_cast<float2*>(at + f.factor_at);
  float2* const stat = reinterpret_cast<float2*>(at + f.stat_at);
  uint16_t* const E = c.grad ? reinterpret_cast<uint16_t*>(at + f.e_at) : nullptr;
  uint16_t* const rows = reinterpret_cast<uint16_t*>(at + f.rows_at);
  float* const part = reinterpret_cast<float*>(at + f.part_at);
  float* const sum = reinterpret_cast<float*>(at + f.sum_at);
  for (int64_t b = 0; b < f.blocks; ++b) {
    const int64_t first = b * f.block, n = c.tokens - first < f.block ? c.tokens - first : f.block;
    const uint16_t* X = static_cast<const uint16_t*>(c.x) + first * c.x_ld;
    const uint16_t* W = static_cast<const uint16_t*>(c.w);
    const ProductForm z = vocab_logits_form(s, n);
    LogitsParams lp{};
    lp.X = X;
    lp.W = W;
    lp.targets = c.targets + first;
    lp.target_z = target_z;
    lp.stat = stat;
    lp.E = E;
    lp.x_ld = c.x_ld;
    lp.w_ld = s.w_ld;
    lp.e_ld = f.e_ld;
    lp.tokens = (int32_t)n;
    lp.vocab = (int32_t)s.vocab;
    lp.hidden = (int32_t)s.hidden;
    lp.e_cols = f.e_cols;
    lp.tiles_m = z.tiles_m;
    lp.tiles_n = z.tiles_n;
    lp.group = z.group;
    lp.chunk = z.chunk;
    lp.scale = s.scale;
    const dim3 grid((unsigned)z.workgroups);
    if (z.tile_m == 64) hipLaunchKernelGGL((logits_kernel<64, 128, 2, 4>), grid, dim3(512), 0, stream, lp);
    else if (z.tile_m == 256) hipLaunchKernelGGL((logits_kernel<256, 256, 2, 4>), grid, dim3(512), 0, stream, lp);
    else hipLaunchKernelGGL((logits_kernel<128, 128, 2, 4>), grid, dim3(512), 0, stream, lp);
    if (hipError_t e = hipGetLastError()) return e;
    CombineParams cp{};
    cp.stat = stat;
    cp.target_z = target_z;
    cp.targets = c.targets + first;
    cp.dloss = c.dloss ? c.dloss + first : nullptr;
    cp.loss = c.loss ? c.loss + first : nullptr;
    cp.lse = c.lse ? c.lse + first : nullptr;
    cp.factor = c.grad ? factor : nullptr;
    cp.tokens = (int32_t)n;
    cp.vocab = (int32_t)s.vocab;
    cp.tiles_n = z.tiles_n;
    cp.scale = s.scale;
    cp.X = X;
    cp.x_ld = c.x_ld;
    cp.rows = c.dw ? rows : nullptr;
    cp.hidden = (int32_t)s.hidden;
    cp.dloss_scale = c.dloss_scale;
    hipLaunchKernelGGL(combine_kernel, dim3((unsigned)((n + 3) / 4)), dim3(256), 0, stream, cp);
    if (hipError_t e = hipGetLastError()) return e;
    if (!c.grad) continue;
    ScaleParams sp{};
    sp.E = E;
    sp.stat = stat;
    sp.factor = factor;
    sp.target_z = target_z;
    sp.targets = c.targets + first;
    sp.e_ld = f.e_ld;
    sp.vocab = (int32_t)s.vocab;
    sp.e_cols = f.e_cols;
    sp.tiles_n = z.tiles_n;
    sp.tile_shift = __builtin_ctz(z.tile_n);
    hipLaunchKernelGGL(scale_kernel, dim3((unsigned)((f.e_cols / 8 + 255) / 256), (unsigned)n), dim3(256), 0, stream, sp);
    if (hipError_t e = hipGetLastError()) return e;
    if (c.dx) {
      const ProductForm d = vocab_dx_form(s, n);
      PlainParams p{};
      p.U = E;
      p.ldu = f.e_ld;
      p.V = W;
      p.ldv = s.w_ld;
      p.m = (int32_t)n;
      p.n = p.nv = (int32_t)s.hidden;
      p.ku = f.e_cols;
      p.kv = (int32_t)s.vocab;
      p.ksteps = f.e_cols / 64;
      p.out = static_cast<uint16_t*>(c.dx) + first * c.dx_ld;
      p.ld_out = c.dx_ld;
      p.part = d.splits > 1 ? part : nullptr;
      if (hipError_t e = launch_plain<true, false>(d, p, stream)) return e;
      if (d.splits > 1) {
        const int64_t elems = n * s.hidden;
        hipLaunchKernelGGL(ranges_kernel, dim3((unsigned)((elems / 4 + 255) / 256)), dim3(256), 0, stream, part, d.splits, elems,
                           (int32_t)s.hidden, static_cast<uint16_t*>(p.out), c.dx_ld);
        if (hipError_t e = hipGetLastError()) return e;
      }
    }
    if (c.dw) {
      PlainParams p{};
      p.U = E;
      p.ldu = f.e_ld;
      p.V = rows;
      p.ldv = s.hidden;
      p.m = (int32_t)s.vocab;
      p.mu = f.e_cols;
      p.n = p.nv = (int32_t)s.hidden;
      p.ku = p.kv = (int32_t)n;
      p.ksteps = (int32_t)((n + 63) / 64);
      // fp32 sums of all blocks but the last: in dW itself, or in the workspace
      const bool last = b + 1 == f.blocks, own = c.dw_f32 || last;
      p.out = own ? c.dw : sum;
      p.ld_out = own ? c.dw_ld : s.hidden;
      p.f32 = c.dw_f32 || !last;
      p.accumulate = c.dw_f32 ? c.accumulate || b > 0 : last ? c.accumulate : b > 0;
      p.add = !c.dw_f32 && last && b > 0 ? sum : nullptr;
      if (hipError_t e = launch_plain<false, false>(vocab_dw_form(s, n), p, stream)) return e;
    }
  }
  return hipSuccess;
}

}  // namespace ccl
