// Experts' products on rows sorted by expert (ccl_grouped_gemm and its
// gradients): expert e has rows ends[e-1] .. ends[e] - 1, its weight is N x K.
//   forward  Z = X W_e^T, Y = act(Z) or act(gate) * up
//   grad     D = dY W_e, dX = D or dZ of X = act(Z), act(gate) * up
//   wgrad    dW_e = dY_e^T X_e (+ dW_e)
// The row counts are on the device only: a launch has as many workgroups as the
// counts can take at most, and each finds its tile from ends by a scan over the
// experts' tiles, one thread an expert.
#include "product.hpp"

#include "train_kernels.hpp"

namespace ccl {

namespace {

struct GroupedParams {
  const uint16_t *U, *V;    // forward X, W; grad dY, W; wgrad dY, X
  const int32_t* ends;
  void* out;
  uint16_t* Z;              // pre-activations: written (forward) or read (grad)
  int64_t ldu, ldv, ld_out, ld_z;
  int64_t w_stride;         // of W, or dW
  int32_t rows, experts, n, k;     // columns of the product, its K (wgrad: rows of dW in n, columns in k)
  int32_t tiles_m, tiles_n, chunk;
  int32_t act, f32, accumulate;
};

// Rows of expert e; whatever ends holds, within 0 .. rows.
__device__ __forceinline__ void expert_rows(const GroupedParams& p, int e, int32_t* first, int32_t* n) {
  const int32_t lo = e ? min(max(p.ends[e - 1], 0), p.rows) : 0, hi = min(max(p.ends[e], 0), p.rows);
  *first = lo;
  *n = max(hi - lo, 0);
}

struct RowTile {
  int32_t expert, first, rows, tj;     // first: row of the tile, rows: of it
};

// Tile `id` of the experts' row tiles, expert by expert, column by column.
template <int BM, int THREADS>
__device__ __forceinline__ bool row_tile(const GroupedParams& p, int64_t id, int32_t* sh, int tid, RowTile* t) {
  const int lane = tid & 63, wave = tid >> 6;
  int32_t first = 0, n = 0;
  if (tid < p.experts) expert_rows(p, tid, &first, &n);
  const int32_t tiles = (n + BM - 1) / BM;
  int32_t sum = tiles;
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) {
    const int32_t other = __shfl_up(sum, x);
    if (lane >= x) sum += other;
  }
  if (lane == 63) sh[wave] = sum;
  __syncthreads();
  int32_t before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) before += sh[w];
    total += sh[w];
  }
  if (id >= (int64_t)total * p.tiles_n) return false;
  const int32_t row = (int32_t)(id / p.tiles_n), from = before + sum - tiles;
  if (row >= from && row < from + tiles) {
    sh[8] = tid;
    sh[9] = from;
    sh[10] = tiles;
    sh[11] = first;
    sh[12] = n;
  }
  __syncthreads();
  const int32_t local = (int32_t)(id - (int64_t)sh[9] * p.tiles_n), of = sh[10];
  const int32_t tj = local / of, ti = local - tj * of;
  t->expert = __builtin_amdgcn_readfirstlane(sh[8]);
  t->first = __builtin_amdgcn_readfirstlane(sh[11] + ti * BM);
  t->rows = __builtin_amdgcn_readfirstlane(min(BM, sh[12] - ti * BM));
  t->tj = __builtin_amdgcn_readfirstlane(tj);
  return true;
}

// Y (and Z) of a tile. A gated tile's columns alternate in groups of 16, gate
// and up, which a lane holds in neighbouring accumulators.
template <typename T, bool GATED>
__device__ __forceinline__ void forward_out(const GroupedParams& p, f32x4 (&acc)[T::TM][T::TN], char* sm, const RowTile& t,
                                            int tid) {
  constexpr int BM = T::BM, BN = T::BN, OUT = GATED ? BN / 2 : BN;
  const int32_t half = p.n / 2;
  uint16_t* const Y = static_cast<uint16_t*>(p.out) + t.first * p.ld_out;
  if (p.Z) {
    const auto z = staged<BM, BN>(sm);
    each4<T>(tid, [&](int mt, int nt, int r, int c) __attribute__((always_inline)) { *z.at(r, c) = f32_to_bf16x4(acc[mt][nt]); });
    staged_barrier();
    tile_out<BM, BN, T::THREADS>(z, p.Z + t.first * p.ld_z, p.ld_z, t.rows, tid, [&](int c) {
      if constexpr (!GATED) return t.tj * BN + 8 * c < p.n ? t.tj * BN + 8 * c : -1;
      const int32_t n = t.tj * OUT + (c >> 2) * 16 + (c & 1) * 8;
      return n < half ? n + (c & 2 ? half : 0) : -1;
    });
    staged_barrier();
  }
  const auto y = staged<BM, OUT>(sm);
  const ActCoef k = act_coef(p.act);
  with_act(p.act, [&](auto cls) __attribute__((always_inline)) {
    constexpr int C = decltype(cls)::value;
    each4<T>(tid, [&](int mt, int nt, int r, int c) __attribute__((always_inline)) {
      if constexpr (GATED) {
        if (nt & 1) return;
        f32x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = act_value<C>(k, acc[mt][nt][j]) * acc[mt][nt + 1][j];
        *y.at(r, (c >> 1 & ~15) + (c & 15)) = f32_to_bf16x4(o);
      } else {
        f32x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = act_value<C>(k, acc[mt][nt][j]);
        *y.at(r, c) = f32_to_bf16x4(o);
      }
    });
  });
  staged_barrier();
  const int32_t cols = GATED ? half : p.n;
  tile_out<BM, OUT, T::THREADS>(y, Y, p.ld_out, t.rows, tid,
                                [&](int c) { return t.tj * OUT + 8 * c < cols ? t.tj * OUT + 8 * c : -1; });
}

// dX or dZ of a tile. Z's gate columns come first, then its up columns, and so
// dZ's.
template <typename T, bool GATED>
__device__ __forceinline__ void grad_out(const GroupedParams& p, f32x4 (&acc)[T::TM][T::TN], char* sm, const RowTile& t,
                                         int tid) {
  constexpr int BM = T::BM, BN = T::BN;
  const auto s = staged<BM, BN>(sm);
  uint16_t* const out = static_cast<uint16_t*>(p.out) + t.first * p.ld_out;
  const uint16_t* const Z = p.Z + t.first * p.ld_z;
  const auto col = [&](int c) { return t.tj * BN + 8 * c < p.n ? t.tj * BN + 8 * c : -1; };
  const auto up_col = [&](int c) { return t.tj * BN + 8 * c < p.n ? p.n + t.tj * BN + 8 * c : -1; };
  const ActCoef k = act_coef(p.act);
  uint2 up[T::TM][T::TN];
  if constexpr (GATED) {
    tile_in<BM, BN, T::THREADS>(s, Z, p.ld_z, t.rows, tid, up_col);
    staged_barrier();
    each4<T>(tid, [&](int mt, int nt, int r, int c) __attribute__((always_inline)) { up[mt][nt] = *s.at(r, c); });
    staged_barrier();
  }
  if (GATED || p.act != ACT_NONE) {
    tile_in<BM, BN, T::THREADS>(s, Z, p.ld_z, t.rows, tid, col);
    staged_barrier();
  }
  with_act(p.act, [&](auto cls) __attribute__((always_inline)) {
    constexpr int C = decltype(cls)::value;
    each4<T>(tid, [&](int mt, int nt, int r, int c) __attribute__((always_inline)) {
      const f32x4 d = acc[mt][nt];
      f32x4 o = d;
      if constexpr (GATED || C != ACT_CLASS_NONE) {
        const f32x4 z = bf16x4_to_f32(*s.at(r, c));
        f32x4 u, w;
        if constexpr (GATED) u = bf16x4_to_f32(up[mt][nt]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float slope;
          const float value = act_value_grad<C>(k, z[j], &slope);
          if constexpr (GATED) {
            w[j] = d[j] * value;
            o[j] = d[j] * u[j] * slope;
          } else {
            o[j] = d[j] * slope;
          }
        }
        if constexpr (GATED) up[mt][nt] = f32_to_bf16x4(w);
      }
      *s.at(r, c) = f32_to_bf16x4(o);
    });
  });
  staged_barrier();
  tile_out<BM, BN, T::THREADS>(s, out, p.ld_out, t.rows, tid, col);
  if constexpr (GATED) {
    staged_barrier();
    each4<T>(tid, [&](int mt, int nt, int r, int c) __attribute__((always_inline)) { *s.at(r, c) = up[mt][nt]; });
    staged_barrier();
    tile_out<BM, BN, T::THREADS>(s, out, p.ld_out, t.rows, tid, up_col);
  }
}

template <int BM, int BN, int NS, int WGN, bool GRAD, bool GATED>
__global__ void __launch_bounds__(512, NS * (BM + BN) * 128 <= 80 * 1024 ? 4 : 2) grouped_rows_kernel(GroupedParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  using T = ProductTile<BM, BN, true, !GRAD, NS, WGN>;
  __shared__ __attribute__((aligned(1024))) char sm[T::LDS];
  const int tid = threadIdx.x;
  RowTile t;
  if (!row_tile<BM, 512>(p, dealt_tile(p.chunk), reinterpret_cast<int32_t*>(sm), tid, &t)) return;
  __syncthreads();
  const uint16_t* W = p.V + t.expert * p.w_stride;
  const Side u{p.U + t.first * p.ldu, p.ldu, t.rows, p.k};
  Side v;
  // a gated tile's V rows: BN / 2 gate rows from row `first` on and the up rows half of the weight later
  constexpr bool kPairs = GATED && !GRAD;
  const int32_t first = kPairs ? t.tj * (BN / 2) : t.tj * BN;
  if constexpr (GRAD) v = Side{W + first, p.ldv, min(BN, p.n - first), p.k};
  else v = Side{W + first * p.ldv, p.ldv, kPairs ? p.n - first : min(BN, p.n - first), p.k};
  const int32_t half = p.n / 2;
  f32x4 acc[T::TM][T::TN];
  product<T>(u, v, 0, (p.k + 63) / 64, acc, sm, tid, [&](int r) {
    if constexpr (!kPairs) return r;
    return (r >> 5) * 16 + (r & 15) + (r & 16 ? half : 0);
  });
  if constexpr (GRAD) grad_out<T, GATED>(p, acc, sm, t, tid);
  else forward_out<T, GATED>(p, acc, sm, t, tid);
#endif
}

// dW tiles: rows of dW from dY's columns, columns from X's, K over the expert's rows.
template <int BM, int BN, int NS, int WGN>
__global__ void __launch_bounds__(512, NS * (BM + BN) * 128 <= 80 * 1024 ? 4 : 2) grouped_wgrad_kernel(GroupedParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  using T = ProductTile<BM, BN, false, false, NS, WGN>;
  __shared__ __attribute__((aligned(1024))) char sm[T::LDS];
  const int tid = threadIdx.x;
  const int64_t id = dealt_tile(p.chunk);
  const int32_t per = p.tiles_m * p.tiles_n;
  if (id >= (int64_t)per * p.experts) return;
  const int32_t e = __builtin_amdgcn_readfirstlane((int32_t)(id / per)), local = (int32_t)(id - (int64_t)e * per);
  const int32_t tj = __builtin_amdgcn_readfirstlane(local / p.tiles_m), ti = local - tj * p.tiles_m;
  int32_t first, rows;
  expert_rows(p, e, &first, &rows);
  first = __builtin_amdgcn_readfirstlane(first);
  rows = __builtin_amdgcn_readfirstlane(rows);
  const int32_t m = min(BM, p.n - ti * BM), n = min(BN, p.k - tj * BN);
  f32x4 acc[T::TM][T::TN];
  if (rows > 0) {
    product<T>(Side{p.U + first * p.ldu + ti * BM, p.ldu, m, rows}, Side{p.V + first * p.ldv + tj * BN, p.ldv, n, rows}, 0,
               (rows + 63) / 64, acc, sm, tid, [](int r) { return r; });
  } else {
    if (p.accumulate) return;
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
      for (int j = 0; j < T::TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int64_t corner = e * p.w_stride + (int64_t)ti * BM * p.ld_out + tj * BN;
  if (p.f32) {
    float* const to = static_cast<float*>(p.out) + corner;
    each4<T>(tid, [&](int mt, int nt, int r, int c) __attribute__((always_inline)) {
      if (r >= m || c >= n) return;
      f32x4* at = reinterpret_cast<f32x4*>(to + r * p.ld_out + c);
      *at = p.accumulate ? *at + acc[mt][nt] : acc[mt][nt];
    });
    return;
  }
  uint16_t* const to = static_cast<uint16_t*>(p.out) + corner;
  const auto s = staged<BM, BN>(sm);
  each4<T>(tid, [&](int mt, int nt, int r, int c) __attribute__((always_inline)) {
    f32x4 o = acc[mt][nt];
    if (p.accumulate && r < m && c < n) o += bf16x4_to_f32(*reinterpret_cast<const uint2*>(to + r * p.ld_out + c));
    *s.at(r, c) = f32_to_bf16x4(o);
  });
  staged_barrier();
  tile_out<BM, BN, T::THREADS>(s, to, p.ld_out, m, tid, [&](int c) { return 8 * c < n ? 8 * c : -1; });
#endif
}

}  // namespace

hipError_t launch_grouped(const GroupedShape& s, const GroupedCall& c, int direction, void* ws, hipStream_t stream) {
  const GroupedForm f = grouped_form(s, c.rows, direction);
  GroupedParams p{};
  p.ends = c.ends;
  p.U = static_cast<const uint16_t*>(c.a);
  p.V = static_cast<const uint16_t*>(c.b);
  p.out = c.out;
  p.Z = static_cast<uint16_t*>(c.z);
  p.ldu = c.a_ld;
  p.ld_out = c.out_ld;
  p.ld_z = c.z_ld;
  p.w_stride = s.w_stride;
  p.rows = (int32_t)c.rows;
  p.experts = s.experts;
  p.tiles_m = f.tiles_m;
  p.tiles_n = f.tiles_n;
  p.chunk = f.chunk;
  p.act = s.act;
  p.f32 = c.f32;
  p.accumulate = c.accumulate;
  const dim3 grid((unsigned)f.workgroups), block(512);
  if (direction == GROUPED_WGRAD) {
    p.ldv = c.b_ld;
    p.ld_out = s.w_ld;
    p.n = (int32_t)s.out;
    p.k = (int32_t)s.in;
    hipLaunchKernelGGL((grouped_wgrad_kernel<128, 128, 2, 4>), grid, block, 0, stream, p);
    return hipGetLastError();
  }
  p.ldv = s.w_ld;
  if (direction == GROUPED_FORWARD) {
    p.n = (int32_t)s.out;
    p.k = (int32_t)s.in;
    if (s.gated) hipLaunchKernelGGL((grouped_rows_kernel<128, 128, 2, 4, false, true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((grouped_rows_kernel<128, 128, 2, 4, false, false>), grid, block, 0, stream, p);
  } else {
    p.n = (int32_t)s.in;
    p.k = (int32_t)s.out;
    if (s.gated) hipLaunchKernelGGL((grouped_rows_kernel<128, 128, 2, 4, true, true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((grouped_rows_kernel<128, 128, 2, 4, true, false>), grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace ccl
