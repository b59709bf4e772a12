// Softmax cross entropy of z = scale X W^T (tokens x vocabulary) against target
// tokens, and its gradients (ccl_cross_entropy, ccl_cross_entropy_grad):
//   lse = log sum_v exp(z_v),  loss = lse - z_t,  p = exp(z - lse)
//   dX = P' W,  dW = P'^T X,  P'_v = g scale (p_v - [v = t])
// for a block of tokens at a time:
//   logits   tiles of X W^T that stay in registers: each leaves the maximum m
//            and sum of exp(z - m) of every row (fp32), the target's z, and for
//            the gradient e = exp(z - m) in 16 bits
//   combine  rows' lse and loss from the tiles' m and sums, in a fixed order
//   scale    e -> P', in place: e exp(m - lse) g scale; the target's p - 1 is
//            expm1(z_t - lse) of the fp32 z_t, since from a rounded p it would
//            lose everything where p is near 1
//   dX, dW   products of P' with W and X
// Logits in fp32 exist nowhere in memory; P' is kept for a block, 2 bytes each,
// so that neither gradient has to recompute them (6 T D V operations rather
// than 8). Rounded: e to 10 significant bits (2^-10 at most), P' to the products' bf16
// (2^-8; the target's from fp32), dX and dW once.
//
// Bound by the matrix cores where there are many tokens: the loss of 4096 tokens, 8192 x
// 32768, 1.60 ms (1.38 PFLOP/s); with both gradients 8192 of 2048 x 131072 11.4 ms: 4.0
// the logits with e's 2.1 GB on their way, 0.68 the scaling (6.3 TB/s), 3.2 dX, 3.4 dW
// (added to in bf16 0.07 more, in fp32 0.14, added to in fp32 0.24; in blocks of 2048
// tokens 13.0 in all, of 1024 14.8: their fp32 sums of dW go in and out).
// One token is W's bytes: 111 us for 2048 x 131072 (4.8 TB/s).
#include <algorithm>

#include "product.hpp"

#include "train_kernels.hpp"

namespace ccl {

namespace {

// e = exp(z - tile maximum) in 16 bits: it is never negative and never above 1, so that
// its fp32's sign and first exponent bit are 0 and 9 bits of mantissa are left beside
// all other exponents (half a step: 2^-10, a quarter of bf16's; sums of P' of tokens that
// are no target are 1.7e-3 from fp32's where bf16 made it 2.2e-3, for 0.1 to 0.5 % more
// time of loss and gradients). Rounded to nearest, two a word. A NaN need not be held:
// its token's lse is NaN.
__device__ __forceinline__ uint32_t held2(float a, float b) {
  const uint32_t x = (__float_as_uint(a) << 2) + 0x8000u, y = (__float_as_uint(b) << 2) + 0x8000u;
  return __builtin_amdgcn_perm(y, x, 0x07060302u);
}
__device__ __forceinline__ float held_low(uint32_t w) { return __uint_as_float((w & 0xffffu) << 14); }
__device__ __forceinline__ float held_high(uint32_t w) { return __uint_as_float((w >> 16) << 14); }

struct LogitsParams {
  const uint16_t *X, *W;
  const int64_t* targets;
  float* target_z;         // [tokens]
  float2* stat;            // [tokens][stat_ld], of these tiles: maximum, sum
  uint16_t* E;             // [tokens][e_ld], or null
  int64_t x_ld, w_ld, e_ld;
  int32_t tokens, vocab, hidden, e_cols;    // vocab, e_cols: from the first column on
  int32_t first, stat_ld;                   // this launch's first column
  int32_t tiles_m, tiles_n, group, chunk;
  float scale;
};

struct LogitsWork {
  Side u, v;
  int32_t steps;
  int32_t ti, tj;
};

template <typename T>
__global__ void __launch_bounds__(T::THREADS, waves_per_simd<T>()) logits_kernel(LogitsParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int BM = T::BM, BN = T::BN, TM = T::TM, TN = T::TN, WGN = T::WGN;
  __shared__ __attribute__((aligned(1024))) char sm[T::LDS];
  __shared__ float part[WGN][BM], whole[BM];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WGN, wn = wave % WGN;
  product_tiles<T, LogitsWork, 0>(
      p.x_ld, p.w_ld, sm, tid,
      [&](int i, LogitsWork* w) __attribute__((always_inline)) {
        const int32_t id = dealt_tile(i, p.chunk);
        if (id >= p.tiles_m * p.tiles_n) return false;
        raster(id, p.tiles_m, p.tiles_n, p.group, &w->ti, &w->tj);
        w->steps = product_steps<T>(p.hidden);
        w->u = Side{p.X + (int64_t)w->ti * BM * p.x_ld, min(BM, p.tokens - w->ti * BM), p.hidden};
        w->v = Side{p.W + (int64_t)w->tj * BN * p.w_ld, min(BN, p.vocab - w->tj * BN), p.hidden};
        return true;
      },
      [](int r) { return r; },
      [&](const LogitsWork& w, f32x4 (&acc)[TM][TN]) __attribute__((always_inline)) {
        const int32_t rows = w.u.extent, col0 = w.tj * BN + wn * T::WN + 4 * (lane >> 4);
        const int32_t left = p.vocab - col0;         // columns from the lane's first on
        const TileMatrix<TN / 2, T::ROWS> E(p.E + (int64_t)w.ti * BM * p.e_ld + w.tj * BN, p.e_ld, p.E ? rows : 0,
                                            p.e_cols - w.tj * BN, T::row(wm, 0) + (lane & 15), wn * T::WN + pair_column(lane));
        // rows' maxima over a wave's columns, then over the waves
        float top[TM], sum[TM];
#pragma unroll
        for (int mt = 0; mt < TM; ++mt) {
          top[mt] = -INFINITY;
          if (T::row(wm, mt) < rows) {
#pragma unroll
            for (int nt = 0; nt < TN; ++nt)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                acc[mt][nt][j] = 16 * nt + j < left ? acc[mt][nt][j] * p.scale : -INFINITY;
                top[mt] = fmaxf(top[mt], acc[mt][nt][j]);
              }
          }
          top[mt] = fmaxf(top[mt], __shfl_xor(top[mt], 16));
          top[mt] = fmaxf(top[mt], __shfl_xor(top[mt], 32));
          if (lane < 16) part[wn][T::row(wm, mt) + lane] = top[mt];
        }
        product_barrier<63>();
#pragma unroll
        for (int mt = 0; mt < TM; ++mt) {
          const int r = T::row(wm, mt) + (lane & 15);
#pragma unroll
          for (int k = 0; k < WGN; ++k) top[mt] = fmaxf(top[mt], part[k][r]);
          if (wn == 0 && lane < 16) whole[r] = top[mt];
          // all of a tile's logits -inf: terms of 0, not of exp(-inf + inf)
          top[mt] = top[mt] == -INFINITY ? 0.f : top[mt];
          sum[mt] = 0.f;
          if (T::row(wm, mt) >= rows) continue;
          // the target's logit
          if (r < rows) {
            const int64_t t = p.targets[w.ti * BM + r] - p.first - col0;
            if (t >= 0 && t < T::WN && t < left) {
#pragma unroll
              for (int nt = 0; nt < TN; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  if (t == 16 * nt + j) p.target_z[w.ti * BM + r] = acc[mt][nt][j];
            }
          }
          uint2 e[TN];
#pragma unroll
          for (int nt = 0; nt < TN; ++nt) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              acc[mt][nt][j] = __builtin_amdgcn_exp2f((acc[mt][nt][j] - top[mt]) * kLog2e);
              sum[mt] += acc[mt][nt][j];
            }
            e[nt] = make_uint2(held2(acc[mt][nt][0], acc[mt][nt][1]), held2(acc[mt][nt][2], acc[mt][nt][3]));
          }
          if (p.E) {
            // columns past the vocabulary up to e_cols: exp(-inf) = 0
#pragma unroll
            for (int i = 0; i < TN / 2; ++i) E.store(mt, i, pair_up(e[2 * i], e[2 * i + 1]));
          }
        }
        product_barrier<63>();
#pragma unroll
        for (int mt = 0; mt < TM; ++mt) {
          sum[mt] += __shfl_xor(sum[mt], 16);
          sum[mt] += __shfl_xor(sum[mt], 32);
          if (lane < 16) part[wn][T::row(wm, mt) + lane] = sum[mt];
        }
        product_barrier<63>();
        if (tid < rows) {
          float s = 0.f;
#pragma unroll
          for (int k = 0; k < WGN; ++k) s += part[k][tid];
          p.stat[(int64_t)(w.ti * BM + tid) * p.stat_ld + w.tj] = make_float2(whole[tid], s);
        }
        // the next tile's finish writes part again
        product_barrier<63>();
      });
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
  int32_t vocab, tiles_n, hidden;
  float scale, dloss_scale;
};

// A workgroup a token: the tiles' sums brought to their common maximum (the same
// order whatever the rest). For dW the tokens' x are copied without those that add
// nothing to it: 0 times whatever a padding row holds need not be 0.
__global__ void __launch_bounds__(256) combine_kernel(CombineParams p) {
  __shared__ float2 waves[4];
  const int32_t row = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const float2* s = p.stat + (int64_t)row * p.tiles_n;
  const int64_t t = p.targets[row];
  const bool live = t >= 0 && t < p.vocab;
  const float g = live ? (p.dloss ? p.dloss[row] : 1.f) * p.dloss_scale * p.scale : 0.f;
  float top = -INFINITY, sum = 0.f;
  const auto join = [&](float2 o) {
    const float m = fmaxf(top, o.x);
    // a side without terms has a maximum of -inf, and 0 terms
    sum = (sum == 0.f ? 0.f : sum * __builtin_amdgcn_exp2f((top - m) * kLog2e)) +
          (o.y == 0.f ? 0.f : o.y * __builtin_amdgcn_exp2f((o.x - m) * kLog2e));
    top = m;
  };
#pragma unroll 4
  for (int i = tid; i < p.tiles_n; i += 256) join(s[i]);
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) join(make_float2(__shfl_xor(top, x), __shfl_xor(sum, x)));
  if (lane == 0) waves[tid >> 6] = make_float2(top, sum);
  if (p.rows) {
    const uint4* from = reinterpret_cast<const uint4*>(p.X + row * p.x_ld);
    uint4* to = reinterpret_cast<uint4*>(p.rows + (int64_t)row * p.hidden);
    for (int i = tid; i < p.hidden / 8; i += 256) to[i] = g != 0.f ? from[i] : make_uint4(0, 0, 0, 0);
  }
  __syncthreads();
  if (tid) return;
  top = waves[0].x;
  sum = waves[0].y;
#pragma unroll
  for (int w = 1; w < 4; ++w) join(waves[w]);
  const float lse = top + logf(sum);
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
  int32_t e_cols, tiles_n;
  int32_t large;           // columns in tiles of 256, the others' are 128 wide
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
  const int32_t tile = col < p.large ? col >> 8 : ((p.large + 255) >> 8) + ((col - p.large) >> 7);
  const float k = __builtin_amdgcn_exp2f((p.stat[(int64_t)row * p.tiles_n + tile].x - f.x) * kLog2e) * f.y;
  f32x4 lo{held_low(e.x), held_high(e.x), held_low(e.y), held_high(e.y)};
  f32x4 hi{held_low(e.z), held_high(e.z), held_low(e.w), held_high(e.w)};
  lo *= k;
  hi *= k;
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
  int32_t m, n, ku, kv;
  int32_t mu, nv;          // columns that U and V have (RC sides, whole 16 bytes)
  int32_t tiles_m, tiles_n, group, chunk, splits, ksplit;
  int32_t f32, accumulate;
};

struct PlainWork {
  Side u, v;
  int32_t steps;
  int32_t ti, tj, split, m, n;
};

// MORE: with what is added, fp32 results and partial sums (apart, since they take
// registers that the 256x256 tiles' loop needs).
template <typename T, bool MORE>
__global__ void __launch_bounds__(T::THREADS, waves_per_simd<T>()) plain_kernel(PlainParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int BM = T::BM, BN = T::BN, TM = T::TM, TN = T::TN;
  __shared__ __attribute__((aligned(1024))) char sm[T::LDS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / T::WGN, wn = wave % T::WGN;
  const int32_t tiles = p.tiles_m * p.tiles_n;
  product_tiles<T, PlainWork, MORE ? 0 : T::TM * T::TN / 2>(
      p.ldu, p.ldv, sm, tid,
      [&](int i, PlainWork* w) __attribute__((always_inline)) {
        const int32_t id = dealt_tile(i, p.chunk);
        if (id >= tiles * p.splits) return false;
        w->split = __builtin_amdgcn_readfirstlane(id / tiles);
        raster(id - w->split * tiles, p.tiles_m, p.tiles_n, p.group, &w->ti, &w->tj);
        // a range ends where the next begins
        const int32_t k0 = w->split * p.ksplit * 64, k = p.ksplit * 64;
        const int32_t ku = min(p.ku - k0, k), kv = min(p.kv - k0, k);
        w->steps = product_steps<T>(max(ku, kv));
        w->m = min(BM, p.m - w->ti * BM);
        w->n = min(BN, p.n - w->tj * BN);
        w->u = T::UK ? Side{p.U + (int64_t)w->ti * BM * p.ldu + k0, w->m, ku}
                     : Side{p.U + (int64_t)k0 * p.ldu + w->ti * BM, min(BM, p.mu - w->ti * BM), ku};
        w->v = T::VK ? Side{p.V + (int64_t)w->tj * BN * p.ldv + k0, w->n, kv}
                     : Side{p.V + (int64_t)k0 * p.ldv + w->tj * BN, min(BN, p.nv - w->tj * BN), kv};
        return true;
      },
      [](int r) { return r; },
      [&](const PlainWork& w, f32x4 (&acc)[TM][TN]) __attribute__((always_inline)) {
        const int64_t row0 = (int64_t)w.ti * BM;
        const int32_t col0 = w.tj * BN;
        const TileMatrix<TN / 2, T::ROWS> out(static_cast<uint16_t*>(p.out) + row0 * p.ld_out + col0, p.ld_out,
                                              p.part || p.f32 ? 0 : w.m, w.n, T::row(wm, 0) + (lane & 15),
                                              wn * T::WN + pair_column(lane));
#pragma unroll
        for (int mt = 0; mt < TM; ++mt) {
          const int r = T::row(wm, mt) + (lane & 15);
          const bool live = r < w.m;
          if (MORE && (p.part || p.f32)) {
            const int64_t at = p.part ? ((int64_t)w.split * p.m + row0 + r) * p.n + col0 : (row0 + r) * p.ld_out + col0;
            float* const to = (p.part ? p.part : static_cast<float*>(p.out)) + at;
#pragma unroll
            for (int nt = 0; nt < TN; ++nt) {
              const int32_t c = wn * T::WN + 16 * nt + 4 * (lane >> 4);
              if (!live || c >= w.n) continue;
              f32x4* const one = reinterpret_cast<f32x4*>(to + c);
              *one = p.accumulate && !p.part ? *one + acc[mt][nt] : acc[mt][nt];
            }
            continue;
          }
          const float* const add = p.add + (row0 + r) * p.n + col0;
#pragma unroll
          for (int i = 0; i < TN / 2; ++i) {
            f32x4 a = acc[mt][2 * i], b = acc[mt][2 * i + 1];
            const int32_t c4 = wn * T::WN + 32 * i + 4 * (lane >> 4);
            if (MORE && p.add && live) {
              if (c4 < w.n) a += *reinterpret_cast<const f32x4*>(add + c4);
              if (c4 + 16 < w.n) b += *reinterpret_cast<const f32x4*>(add + c4 + 16);
            }
            if (MORE && p.accumulate) {
              uint2 x, y;
              pair_down(out.load(mt, i), &x, &y);
              a += bf16x4_to_f32(x);
              b += bf16x4_to_f32(y);
            }
            out.store(mt, i, pair_up(f32_to_bf16x4(a), f32_to_bf16x4(b)));
          }
        }
      });
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
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < rows * row_chunks; at += (int64_t)gridDim.x * 256) {
    const int64_t r = at / row_chunks;
    *reinterpret_cast<uint4*>(out + r * ld_bytes + (at - r * row_chunks) * 16) = make_uint4(0, 0, 0, 0);
  }
}

template <bool UK, bool VK>
hipError_t launch_plain(const ProductForm& f, PlainParams p, hipStream_t stream) {
  p.tiles_m = f.tiles_m;
  p.tiles_n = f.tiles_n;
  p.group = f.group;
  p.chunk = f.chunk;
  p.splits = f.splits;
  p.ksplit = f.ksplit;
  const auto launch = [&](auto tile) {
    using T = decltype(tile);
    if (p.part || p.f32 || p.add || p.accumulate)
      hipLaunchKernelGGL((plain_kernel<T, true>), dim3((unsigned)f.workgroups), dim3(T::THREADS), 0, stream, p);
    else
      hipLaunchKernelGGL((plain_kernel<T, false>), dim3((unsigned)f.workgroups), dim3(T::THREADS), 0, stream, p);
  };
  if (f.tile_m == 256) launch(ProductTile<256, 256, UK, VK, 2, 8, 4, false, true>{});     // KC: columns of P', whole 64s
  else if (f.tile_m == 128) launch(ProductTile<128, 128, UK, VK, 2, 8, 2>{});
  else if constexpr (UK) launch(ProductTile<64, 128, UK, VK, 2, 8, 2, true>{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cross_entropy(const VocabShape& s, const VocabCall& c, void* ws, hipStream_t stream) {
  if (c.tokens == 0) {
    if (!c.grad || !c.dw || c.accumulate) return hipSuccess;
    const int64_t size = c.dw_f32 ? 4 : 2, chunks = s.hidden * size / 16;
    hipLaunchKernelGGL(zero_kernel, dim3((unsigned)std::min<int64_t>((s.vocab * chunks + 255) / 256, 65536)), dim3(256), 0,
                       stream, static_cast<char*>(c.dw), s.vocab, chunks, c.dw_ld * size);
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
    const int64_t large = vocab_logits_large(s, n);
    const int32_t tiles_n = (int32_t)((large + 255) / 256 + (s.vocab - large + 127) / 128);
    LogitsParams lp{};
    lp.X = X;
    lp.targets = c.targets + first;
    lp.target_z = target_z;
    lp.x_ld = c.x_ld;
    lp.w_ld = s.w_ld;
    lp.e_ld = f.e_ld;
    lp.tokens = (int32_t)n;
    lp.hidden = (int32_t)s.hidden;
    lp.scale = s.scale;
    lp.stat_ld = tiles_n;
    ProductForm z;
    const auto logits = [&](auto tile) {
      using T = decltype(tile);
      hipLaunchKernelGGL(logits_kernel<T>, dim3((unsigned)z.workgroups), dim3(T::THREADS), 0, stream, lp);
    };
    // columns `from` to `to` - 1, tiles `nth` on of a row's
    const auto part_of = [&](int64_t from, int64_t to, int64_t nth) {
      z = vocab_logits_form(s, n, to - from, to <= large);
      lp.W = W + from * s.w_ld;
      lp.E = E ? E + from : nullptr;
      lp.first = (int32_t)from;
      lp.stat = stat + nth;
      lp.vocab = (int32_t)(to - from);
      lp.e_cols = (int32_t)((to < s.vocab ? to : f.e_cols) - from);
      lp.tiles_m = z.tiles_m;
      lp.tiles_n = z.tiles_n;
      lp.group = z.group;
      lp.chunk = z.chunk;
      if (z.tile_m == 256 && s.hidden % 64 == 0) logits(ProductTile<256, 256, true, true, 2, 8, 4, false, true>{});
      else if (z.tile_m == 256) logits(ProductTile<256, 256, true, true, 2, 8, 4>{});
      else if (z.tile_m == 128 && z.tiles <= 256) logits(ProductTile<128, 128, true, true, 4, 8, 2>{});
      else if (z.tile_m == 128) logits(ProductTile<128, 128, true, true, 2, 8, 2>{});
      else logits(ProductTile<64, 128, true, true, 3, 8, 2, true>{});
      return hipGetLastError();
    };
    if (large)
      if (hipError_t e = part_of(0, large, 0)) return e;
    if (large < s.vocab)
      if (hipError_t e = part_of(large, s.vocab, (large + 255) / 256)) return e;
    CombineParams cp{};
    cp.stat = stat;
    cp.target_z = target_z;
    cp.targets = c.targets + first;
    cp.dloss = c.dloss ? c.dloss + first : nullptr;
    cp.loss = c.loss ? c.loss + first : nullptr;
    cp.lse = c.lse ? c.lse + first : nullptr;
    cp.factor = c.grad ? factor : nullptr;
    cp.vocab = (int32_t)s.vocab;
    cp.tiles_n = tiles_n;
    cp.scale = s.scale;
    cp.X = X;
    cp.x_ld = c.x_ld;
    cp.rows = c.dw ? rows : nullptr;
    cp.hidden = (int32_t)s.hidden;
    cp.dloss_scale = c.dloss_scale;
    hipLaunchKernelGGL(combine_kernel, dim3((unsigned)n), dim3(256), 0, stream, cp);
    if (hipError_t e = hipGetLastError()) return e;
    if (!c.grad) continue;
    ScaleParams sp{};
    sp.E = E;
    sp.stat = stat;
    sp.factor = factor;
    sp.target_z = target_z;
    sp.targets = c.targets + first;
    sp.e_ld = f.e_ld;
    sp.e_cols = f.e_cols;
    sp.tiles_n = tiles_n;
    sp.large = large < s.vocab ? (int32_t)large : f.e_cols;
    hipLaunchKernelGGL(scale_kernel, dim3((unsigned)((f.e_cols / 8 + 255) / 256), (unsigned)n), dim3(256), 0, stream, sp);
    if (hipError_t e = hipGetLastError()) return e;
    if (c.dx) {
      PlainParams p{};
      p.ldu = f.e_ld;
      p.V = W;
      p.ldv = s.w_ld;
      p.n = p.nv = (int32_t)s.hidden;
      p.ku = f.e_cols;
      p.kv = (int32_t)s.vocab;
      p.ld_out = c.dx_ld;
      const int64_t whole = vocab_dx_large(s, n);
      const auto rows_of = [&](int64_t from, int64_t to) {
        const ProductForm d = vocab_dx_form(s, to - from, to <= whole);
        uint16_t* const out = static_cast<uint16_t*>(c.dx) + (first + from) * c.dx_ld;
        p.U = E + from * f.e_ld;
        p.m = (int32_t)(to - from);
        p.out = out;
        p.part = d.splits > 1 ? part : nullptr;
        const hipError_t e = launch_plain<true, false>(d, p, stream);
        if (e || d.splits == 1) return e;
        const int64_t elems = (to - from) * s.hidden;
        hipLaunchKernelGGL(ranges_kernel, dim3((unsigned)((elems / 4 + 255) / 256)), dim3(256), 0, stream, part, d.splits, elems,
                           (int32_t)s.hidden, out, c.dx_ld);
        return hipGetLastError();
      };
      if (whole)
        if (hipError_t e = rows_of(0, whole)) return e;
      if (whole < n)
        if (hipError_t e = rows_of(whole, n)) return e;
    }
    if (c.dw) {
      PlainParams p{};
      p.ldu = f.e_ld;
      p.V = rows;
      p.ldv = s.hidden;
      p.n = p.nv = (int32_t)s.hidden;
      p.ku = p.kv = (int32_t)n;
      // fp32 sums of all blocks but the last: in dW itself, or in the workspace
      const bool last = b + 1 == f.blocks, own = c.dw_f32 || last;
      p.out = own ? c.dw : sum;
      p.ld_out = own ? c.dw_ld : s.hidden;
      p.f32 = c.dw_f32 || !last;
      p.accumulate = c.dw_f32 ? c.accumulate || b > 0 : last ? c.accumulate : b > 0;
      p.add = !c.dw_f32 && last && b > 0 ? sum : nullptr;
      const int64_t whole = vocab_dw_large(s, n), size = p.f32 ? 4 : 2;
      const auto rows_of = [&](int64_t from, int64_t to) {
        PlainParams q = p;
        q.U = E + from;
        q.m = (int32_t)(to - from);
        q.mu = (int32_t)(f.e_cols - from);
        q.out = static_cast<char*>(p.out) + from * p.ld_out * size;
        q.add = p.add ? p.add + from * s.hidden : nullptr;
        return launch_plain<false, false>(vocab_dw_form(s, n, to - from, to <= whole), q, stream);
      };
      if (whole)
        if (hipError_t e = rows_of(0, whole)) return e;
      if (whole < s.vocab)
        if (hipError_t e = rows_of(whole, s.vocab)) return e;
    }
  }
  return hipSuccess;
}

}  // namespace ccl
