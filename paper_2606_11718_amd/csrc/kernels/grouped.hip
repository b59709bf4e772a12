// Experts' products on rows sorted by expert (ccl_grouped_gemm and its
// gradients): expert e has rows ends[e-1] .. ends[e] - 1, its weight is N x K.
//   forward  Z = X W_e^T, Y = act(Z) or act(gate) * up
//   grad     D = dY W_e, dX = D or dZ of X = act(Z), act(gate) * up
//   wgrad    dW_e = dY_e^T X_e (+ dW_e)
// The row counts are on the device only: every workgroup makes a table of the
// experts' rows and tiles in LDS and takes its tiles from it. Each weight is read by
// the row tiles of its expert, which run next to each other on one XCD.
//
// What bounds them (MI355X): 256 rows an expert are about as many operations as bytes
// (1.09 GB and 206 GFLOP forward), and a tile of 4 to 32 steps spends as long on its
// first loads, its last rows and its stores as on its products. 32768 rows over 128
// experts: 2048 -> 2 x 768 through SwiGLU with Z kept 326 us (3.3 TB/s, 0.63 PFLOP/s),
// its down projection's gradient 205 us (3.6 TB/s), dW of 1536 x 2048 368 us (2.8 TB/s);
// 800 rows over 128 of 768 -> 2048 74 us (5.5 TB/s, as a copy). dW of one row an
// expert, which is its stores alone, takes 160 us, and each 64 rows more 45 to 65:
// loads wait behind the stores of the tile before. Without an activation: forward of 768
// -> 2048 181 us (3.3 TB/s), gradient of 1536 -> 2048 341 us (3.1 TB/s). dW of 1536 x
// 2048 added to in bf16 495 us (3.7 TB/s), in fp32 560 (3.3), added to in fp32 748 (4.6).
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
  int32_t splits;           // K ranges of a tile
  float* part;              // with ranges: their fp32 products, [splits][rows (wgrad: dW's)][columns]
  int32_t act, f32, accumulate;
};

// Each expert's first row, rows, and row tiles of the experts before it.
struct ExpertTable {
  int32_t first[kGroupedMaxExperts], rows[kGroupedMaxExperts], before[kGroupedMaxExperts];
  int32_t total;
  int32_t order[64];       // of up to 64 experts: those with more rows first
};

// The sum or maximum over a wave's lanes before a lane and its own.
template <typename F>
__device__ __forceinline__ int32_t wave_scan(int32_t v, int lane, F&& f) {
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) {
    const int32_t other = __shfl_up(v, x);
    if (lane >= x) v = f(v, other);
  }
  return v;
}

// The table for tiles of BM rows, made by the first wave; the number of row tiles.
// Whatever ends holds, the experts' rows lie one behind the other within 0 ..
// p.rows: the tiles are as many as the launch expects at most, and inside the
// matrices.
template <int BM>
__device__ __forceinline__ int32_t make_table(const GroupedParams& p, ExpertTable& t, int tid) {
  if (tid < 64) {
    int32_t end[kGroupedMaxExperts / 64];
#pragma unroll
    for (int i = 0; i < kGroupedMaxExperts / 64; ++i)
      end[i] = 64 * i + tid < p.experts ? min(max(p.ends[64 * i + tid], 0), p.rows) : 0;
    int32_t past = 0, before = 0;       // of the experts so far
    int32_t mine = 0;                   // the rows of expert tid
#pragma unroll
    for (int i = 0; i < kGroupedMaxExperts / 64; ++i) {
      if (64 * i >= p.experts) break;
      const int32_t to = max(past, wave_scan(end[i], tid, [](int32_t a, int32_t b) { return max(a, b); }));
      const int32_t prev = __shfl_up(to, 1), first = tid ? prev : past;
      const int32_t tiles = (to - first + BM - 1) / BM;
      const int32_t sum = before + wave_scan(tiles, tid, [](int32_t a, int32_t b) { return a + b; });
      t.first[64 * i + tid] = first;
      t.rows[64 * i + tid] = to - first;
      if (i == 0) mine = to - first;
      t.before[64 * i + tid] = sum - tiles;
      past = __shfl(to, 63);
      before = __shfl(sum, 63);
    }
    if (tid == 0) t.total = before;
    if (p.experts <= 64) {
      // from lane to lane: no lane reads what another one has written to the table before the barrier
      int32_t rank = 0;
      for (int e = 0; e < p.experts; ++e) {
        const int32_t other = __builtin_amdgcn_readlane(mine, e);
        rank += other > mine || (other == mine && e < tid);
      }
      if (tid < p.experts) t.order[rank] = tid;
    }
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(t.total);
}

// The last expert with at most `row` row tiles before it: the one that has it.
__device__ __forceinline__ int32_t expert_of(const ExpertTable& t, int32_t experts, int32_t row, int lane) {
  int32_t count = 0;
  for (int e = 0; e < experts; e += 64)
    count += __popcll(__ballot(e + lane < experts && t.before[e + lane] <= row));
  return __builtin_amdgcn_readfirstlane(count - 1);
}

// 256x256 tiles are taken where they fill the CUs: their K is never in ranges.
template <typename T>
constexpr bool kRanges = T::BM < 256;

struct RowWork {
  Side u, v;
  int32_t steps;
  int32_t first, rows, tj;     // rows of the matrices, column tile
  int32_t split;
};

// A range of a tile's K in fp32: one row of it at `to`, columns < n.
template <typename T, typename Col>
__device__ __forceinline__ void partial_row(float* to, const f32x4 (&acc)[T::TN], bool live, int32_t n, int wn, int lane, Col&& col) {
#pragma unroll
  for (int nt = 0; nt < T::TN; ++nt) {
    const int32_t c = col(wn * T::WN + 16 * nt) + 4 * (lane >> 4);
    if (live && c < n) *reinterpret_cast<f32x4*>(to + c) = acc[nt];
  }
}

// Y (and Z) of a tile. A gated tile's columns alternate in groups of 16, gate
// and up, which a lane holds in neighbouring accumulators.
template <typename T, bool GATED>
__device__ __forceinline__ void forward_out(const GroupedParams& p, const RowWork& t, f32x4 (&acc)[T::TM][T::TN], int tid) {
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / T::WGN, wn = wave % T::WGN;
  constexpr int TY = GATED ? T::TN / 2 : T::TN, kHalf = GATED ? 2 : 1;
  static_assert(TY % 2 == 0, "pairs");
  const int32_t cols = p.n / kHalf, corner = t.tj * T::BN / kHalf;      // of Y
  const int row0 = T::row(wm, 0) + (lane & 15);
  const TileMatrix<TY / 2, T::ROWS> Y(static_cast<uint16_t*>(p.out) + t.first * p.ld_out + corner, p.ld_out, t.rows,
                                      cols - corner, row0, wn * T::WN / kHalf + pair_column(lane));
  const ActCoef k = act_coef(p.act);
  if (p.Z) {
    const uint16_t* const z = p.Z + t.first * p.ld_z + corner;
    // gated: even 16s of lanes hold a pair's gate columns and odd ones its up columns,
    // half a Z further on; pairs are 16 columns apart
    const int32_t half = GATED && lane & 16 ? cols : 0;
    TileMatrix<T::TN / 2, T::ROWS> Z(z, p.ld_z, t.rows, GATED ? p.n - corner : cols - corner, row0,
                                     wn * T::WN / kHalf + (GATED ? 8 * (lane >> 5) + half : pair_column(lane)));
    if constexpr (GATED) {
#pragma unroll
      for (int i = 0; i < T::TN / 2; ++i) {
        const int32_t c = wn * T::WN / 2 + 8 * (lane >> 5) + 16 * i;
        Z.at[i] = c < cols - corner ? (uint32_t)(row0 * (int32_t)p.ld_z + c + half) * 2u : 0x80000000u;
      }
    }
#pragma unroll
    for (int mt = 0; mt < T::TM; ++mt) {
      if (T::row(wm, mt) >= t.rows) break;
#pragma unroll
      for (int i = 0; i < T::TN / 2; ++i) Z.store(mt, i, pair_up(f32_to_bf16x4(acc[mt][2 * i]), f32_to_bf16x4(acc[mt][2 * i + 1])));
    }
  }
  with_act(p.act, [&](auto cls) __attribute__((always_inline)) {
    constexpr int C = decltype(cls)::value;
#pragma unroll
    for (int mt = 0; mt < T::TM; ++mt) {
      if (T::row(wm, mt) >= t.rows) break;
      uint2 y[TY];
#pragma unroll
      for (int i = 0; i < TY; ++i) {
        f32x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          o[j] = act_value<C>(k, acc[mt][kHalf * i][j]);
          if constexpr (GATED) o[j] *= acc[mt][2 * i + 1][j];
        }
        y[i] = f32_to_bf16x4(o);
      }
#pragma unroll
      for (int i = 0; i < TY / 2; ++i) Y.store(mt, i, pair_up(y[2 * i], y[2 * i + 1]));
    }
  });
}

// dX or dZ of a tile. Z's gate columns come first, then its up columns, and so
// dZ's.
template <typename T, bool GATED>
__device__ __forceinline__ void grad_out(const GroupedParams& p, const RowWork& t, f32x4 (&acc)[T::TM][T::TN], int tid) {
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / T::WGN, wn = wave % T::WGN;
  constexpr int TP = T::TN / 2;
  const int32_t corner = t.tj * T::BN, cols = p.n - corner;
  const int row0 = T::row(wm, 0) + (lane & 15), col0 = wn * T::WN + pair_column(lane);
  uint16_t* const o = static_cast<uint16_t*>(p.out) + t.first * p.ld_out + corner;
  const uint16_t* const z = p.Z + t.first * p.ld_z + corner;
  using Matrix = TileMatrix<TP, T::ROWS>;
  const Matrix out(o, p.ld_out, t.rows, cols, row0, col0);
  const ActCoef k = act_coef(p.act);
  with_act(p.act, [&](auto cls) __attribute__((always_inline)) {
    constexpr int C = decltype(cls)::value;
    if constexpr (!GATED && C == ACT_CLASS_NONE) {
#pragma unroll
      for (int mt = 0; mt < T::TM; ++mt) {
        if (T::row(wm, mt) >= t.rows) break;
#pragma unroll
        for (int i = 0; i < TP; ++i) out.store(mt, i, pair_up(f32_to_bf16x4(acc[mt][2 * i]), f32_to_bf16x4(acc[mt][2 * i + 1])));
      }
    } else {
      const Matrix out_up(o + p.n, p.ld_out, GATED ? t.rows : 0, cols, row0, col0);
      const Matrix Z(z, p.ld_z, t.rows, cols, row0, col0), Z_up(z + p.n, p.ld_z, GATED ? t.rows : 0, cols, row0, col0);
      // Z of one row of 16x16 tiles is on its way while the one before is worked on
      uint4 zg[2][TP], zu[2][TP];
      auto fetch = [&](int mt) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < TP; ++i) {
          zg[mt & 1][i] = Z.load(mt, i);
          if constexpr (GATED) zu[mt & 1][i] = Z_up.load(mt, i);
        }
      };
      fetch(0);
#pragma unroll
      for (int mt = 0; mt < T::TM; ++mt) {
        if (T::row(wm, mt) >= t.rows) break;
        if (mt + 1 < T::TM) fetch(mt + 1);
#pragma unroll
        for (int i = 0; i < TP; ++i) {
          uint2 x[2], w[2], g[2], u[2];
          pair_down(zg[mt & 1][i], &g[0], &g[1]);
          if constexpr (GATED) pair_down(zu[mt & 1][i], &u[0], &u[1]);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const f32x4 d = acc[mt][2 * i + h], gate = bf16x4_to_f32(g[h]);
            f32x4 dg, du, up;
            if constexpr (GATED) up = bf16x4_to_f32(u[h]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float slope;
              const float value = act_value_grad<C>(k, gate[j], &slope);
              if constexpr (GATED) {
                du[j] = d[j] * value;
                dg[j] = d[j] * up[j] * slope;
              } else {
                dg[j] = d[j] * slope;
              }
            }
            x[h] = f32_to_bf16x4(dg);
            if constexpr (GATED) w[h] = f32_to_bf16x4(du);
          }
          out.store(mt, i, pair_up(x[0], x[1]));
          if constexpr (GATED) out_up.store(mt, i, pair_up(w[0], w[1]));
        }
      }
    }
  });
}

template <typename T, bool GRAD, bool GATED>
__global__ void __launch_bounds__(T::THREADS, waves_per_simd<T>()) grouped_rows_kernel(GroupedParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(65536))) char sm[T::LDS];
  __shared__ ExpertTable table;
  const int tid = threadIdx.x, lane = tid & 63;
  const int32_t tiles = make_table<T::BM>(p, table, tid) * p.tiles_n;
  // a gated tile's V rows: BN / 2 gate rows from row `from` on and the up rows half of the weight later
  constexpr bool kPairs = GATED && !GRAD;
  const int32_t half = p.n / 2;
  product_tiles<T, RowWork, 0>(
      p.ldu, p.ldv, sm, tid,
      [&](int i, RowWork* w) __attribute__((always_inline)) {
        int32_t id = dealt_tile(i, p.chunk);
        if (id >= (kRanges<T> ? tiles * p.splits : tiles)) return false;
        w->split = 0;
        int32_t k0 = 0, k = p.k;
        if (kRanges<T> && p.splits > 1) {
          w->split = __builtin_amdgcn_readfirstlane(id / tiles);
          id -= w->split * tiles;
          const int32_t per = ((p.k + 63) / 64 + p.splits - 1) / p.splits * 64;
          k0 = __builtin_amdgcn_readfirstlane(w->split * per);
          k = __builtin_amdgcn_readfirstlane(max(min(per, p.k - k0), 0));
        }
        const int32_t e = expert_of(table, p.experts, __builtin_amdgcn_readfirstlane(id / p.tiles_n), lane);
        const int32_t rows = __builtin_amdgcn_readfirstlane(table.rows[e]), of = (rows + T::BM - 1) / T::BM;
        const int32_t local = id - __builtin_amdgcn_readfirstlane(table.before[e]) * p.tiles_n;
        const int32_t tj = __builtin_amdgcn_readfirstlane(local / of), ti = local - tj * of;
        w->tj = tj;
        w->first = __builtin_amdgcn_readfirstlane(table.first[e]) + ti * T::BM;
        w->rows = min(T::BM, rows - ti * T::BM);
        w->steps = product_steps<T>(k);
        w->u = Side{p.U + w->first * p.ldu + k0, w->rows, k};
        const int32_t from = kPairs ? tj * (T::BN / 2) : tj * T::BN;
        const uint16_t* W = p.V + e * p.w_stride;
        w->v = GRAD ? Side{W + k0 * p.ldv + from, min(T::BN, p.n - from), k}
                    : Side{W + from * p.ldv + k0, kPairs ? p.n - from : min(T::BN, p.n - from), k};
        return true;
      },
      [&](int r) __attribute__((always_inline)) { return kPairs ? (r >> 5) * 16 + (r & 15) + (r & 16 ? half : 0) : r; },
      [&](const RowWork& w, f32x4 (&acc)[T::TM][T::TN]) __attribute__((always_inline)) {
        if (kRanges<T> && p.part) {
          const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / T::WGN, wn = wave % T::WGN;
#pragma unroll
          for (int mt = 0; mt < T::TM; ++mt) {
            const int r = T::row(wm, mt) + (lane & 15);
            float* const to = p.part + ((int64_t)w.split * p.rows + w.first + r) * p.n;
            if constexpr (kPairs) {
              // tile columns alternate, 16 gate and 16 up ones
              partial_row<T>(to, acc[mt], r < w.rows, p.n, wn, lane, [&](int c) {
                const int32_t n = w.tj * (T::BN / 2) + c / 2 - (c & 16) / 2;
                return n >= half ? p.n : n + (c & 16 ? half : 0);
              });
            } else {
              partial_row<T>(to, acc[mt], r < w.rows, p.n, wn, lane, [&](int c) { return w.tj * T::BN + c; });
            }
          }
          return;
        }
        if constexpr (GRAD) grad_out<T, GATED>(p, w, acc, tid);
        else forward_out<T, GATED>(p, w, acc, tid);
      });
#endif
}

struct WgradWork {
  Side u, v;
  int32_t steps;
  int32_t m, n;                // of the tile
  int32_t row, col;            // its corner, row of all experts' dW
  int32_t split, expert;
};

// dW tiles: rows of dW from dY's columns, columns from X's, K over the expert's rows.
// What is done with a tile is a kernel of its own each, since together they take
// registers that the 256x256 tiles' loop needs.
enum WgradOut { WGRAD_BF16, WGRAD_F32, WGRAD_ANY };
template <typename T, WgradOut OUT>
__global__ void __launch_bounds__(T::THREADS, waves_per_simd<T>()) grouped_wgrad_kernel(GroupedParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(65536))) char sm[T::LDS];
  __shared__ ExpertTable table;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  make_table<T::BM>(p, table, tid);
  const int32_t per = p.tiles_m * p.tiles_n;
  const int32_t tiles = per * p.experts;
  product_tiles<T, WgradWork, OUT == WGRAD_BF16 ? T::TM * T::TN / 2 : 0>(
      p.ldu, p.ldv, sm, tid,
      [&](int i, WgradWork* w) __attribute__((always_inline)) {
        int32_t id = dealt_tile(i, p.chunk);
        if (id >= tiles * p.splits) return false;
        w->split = __builtin_amdgcn_readfirstlane(p.splits > 1 ? id / tiles : 0);
        id -= w->split * tiles;
        // few experts' tiles are few for a workgroup: the longest first
        const int32_t nth = __builtin_amdgcn_readfirstlane(id / per), local = id - nth * per;
        const int32_t e = p.experts <= 64 ? __builtin_amdgcn_readfirstlane(table.order[nth]) : nth;
        const int32_t tj = __builtin_amdgcn_readfirstlane(local / p.tiles_m), ti = local - tj * p.tiles_m;
        int32_t first = __builtin_amdgcn_readfirstlane(table.first[e]), rows = __builtin_amdgcn_readfirstlane(table.rows[e]);
        if (p.splits > 1) {
          const int32_t range = ((rows + 63) / 64 + p.splits - 1) / p.splits * 64;
          const int32_t k0 = __builtin_amdgcn_readfirstlane(min(w->split * range, rows));
          first += k0;
          rows = __builtin_amdgcn_readfirstlane(min(range, rows - k0));
        }
        w->m = min(T::BM, p.n - ti * T::BM);
        w->n = min(T::BN, p.k - tj * T::BN);
        w->steps = product_steps<T>(rows);
        w->u = Side{p.U + first * p.ldu + ti * T::BM, w->m, rows};
        w->v = Side{p.V + first * p.ldv + tj * T::BN, w->n, rows};
        w->row = ti * T::BM;
        w->col = tj * T::BN;
        w->expert = e;
        return true;
      },
      [](int r) { return r; },
      [&](const WgradWork& w, f32x4 (&acc)[T::TM][T::TN]) __attribute__((always_inline)) {
        const int wm = wave / T::WGN, wn = wave % T::WGN;
        const int64_t corner = w.expert * p.w_stride + (int64_t)w.row * p.ld_out + w.col;
        const TileMatrix<T::TN / 2, T::ROWS> dw(static_cast<uint16_t*>(p.out) + corner, p.ld_out,
                                                p.f32 || p.part ? 0 : w.m, w.n, T::row(wm, 0) + (lane & 15),
                                                wn * T::WN + pair_column(lane));
#pragma unroll
        for (int mt = 0; mt < T::TM; ++mt) {
          const int r = T::row(wm, mt) + (lane & 15);
          const bool live = r < w.m;
          if (kRanges<T> && OUT == WGRAD_ANY && p.part) {
            float* const to = p.part + (((int64_t)w.split * p.experts + w.expert) * p.n + w.row + r) * p.k + w.col;
            partial_row<T>(to, acc[mt], live, w.n, wn, lane, [](int c) { return c; });
            continue;
          }
          if (OUT == WGRAD_F32 || (OUT == WGRAD_ANY && p.f32)) {
            float* const to = static_cast<float*>(p.out) + corner + r * p.ld_out;
#pragma unroll
            for (int nt = 0; nt < T::TN; ++nt) {
              const int32_t c = wn * T::WN + 16 * nt + 4 * (lane >> 4);
              if (!live || c >= w.n) continue;
              f32x4* at = reinterpret_cast<f32x4*>(to + c);
              *at = OUT == WGRAD_ANY && p.accumulate ? *at + acc[mt][nt] : acc[mt][nt];
            }
          } else {
#pragma unroll
            for (int i = 0; i < T::TN / 2; ++i) {
              f32x4 a = acc[mt][2 * i], b = acc[mt][2 * i + 1];
              if (OUT == WGRAD_ANY && p.accumulate) {
                uint2 x, y;
                pair_down(dw.load(mt, i), &x, &y);
                a += bf16x4_to_f32(x);
                b += bf16x4_to_f32(y);
              }
              dw.store(mt, i, pair_up(f32_to_bf16x4(a), f32_to_bf16x4(b)));
            }
          }
        }
      });
#endif
}

// The ranges' sums in order and what their product's finish does, eight columns a
// thread: FORWARD of Y, GRAD of dX, WGRAD of dW.
template <int DIRECTION, bool GATED>
__global__ void __launch_bounds__(256) grouped_sum_kernel(GroupedParams p) {
  constexpr bool kForward = DIRECTION == GROUPED_FORWARD;
  const int32_t cols = DIRECTION == GROUPED_WGRAD ? p.k : p.n, half = p.n / 2, out = kForward && GATED ? half : cols;
  const int32_t width = out / 8;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, all = DIRECTION == GROUPED_WGRAD ? (int64_t)p.experts * p.n : p.rows;
  const int64_t r = at / width;
  const int32_t c = (int32_t)(at - r * width) * 8;
  if (r >= all) return;
  if constexpr (DIRECTION != GROUPED_WGRAD) {
    // rows behind the last expert's were not computed and stay as they are
    int32_t end = 0;
    for (int e = 0; e < p.experts; ++e) end = max(end, p.ends[e]);
    if (r >= end) return;
  }
  const auto sum8 = [&](int32_t col, f32x4 (&v)[2]) {
    v[0] = v[1] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float* from = p.part + r * cols + col;
#pragma unroll 4
    for (int32_t i = 0; i < p.splits; ++i) {
      v[0] += reinterpret_cast<const f32x4*>(from + i * all * cols)[0];
      v[1] += reinterpret_cast<const f32x4*>(from + i * all * cols)[1];
    }
  };
  const auto store8 = [](uint16_t* to, const f32x4 (&v)[2]) {
    const uint2 a = f32_to_bf16x4(v[0]), b = f32_to_bf16x4(v[1]);
    *reinterpret_cast<uint4*>(to) = make_uint4(a.x, a.y, b.x, b.y);
  };
  const auto load8 = [](const uint16_t* from, f32x4 (&v)[2]) {
    const uint4 a = *reinterpret_cast<const uint4*>(from);
    v[0] = bf16x4_to_f32(make_uint2(a.x, a.y));
    v[1] = bf16x4_to_f32(make_uint2(a.z, a.w));
  };
  f32x4 v[2], u[2];
  sum8(c, v);
  if constexpr (DIRECTION == GROUPED_WGRAD) {
    const int64_t e = r / p.n, to = e * p.w_stride + (r - e * p.n) * p.ld_out + c;
    if (p.f32) {
      f32x4* const dst = reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + to);
#pragma unroll
      for (int i = 0; i < 2; ++i) dst[i] = p.accumulate ? dst[i] + v[i] : v[i];
    } else {
      uint16_t* const dst = static_cast<uint16_t*>(p.out) + to;
      if (p.accumulate) {
        load8(dst, u);
        v[0] += u[0];
        v[1] += u[1];
      }
      store8(dst, v);
    }
    return;
  }
  const ActCoef k = act_coef(p.act);
  uint16_t* const to = static_cast<uint16_t*>(p.out) + r * p.ld_out + c;
  uint16_t* const Z = p.Z + r * p.ld_z + c;
  with_act(p.act, [&](auto cls) __attribute__((always_inline)) {
    constexpr int C = decltype(cls)::value;
    if constexpr (kForward) {
      if constexpr (GATED) sum8(half + c, u);
      if (p.Z) {
        store8(Z, v);
        if constexpr (GATED) store8(Z + half, u);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i >> 2][i & 3] = act_value<C>(k, v[i >> 2][i & 3]);
        if constexpr (GATED) v[i >> 2][i & 3] *= u[i >> 2][i & 3];
      }
    } else if constexpr (GATED || C != ACT_CLASS_NONE) {
      f32x4 z[2], y[2];
      load8(Z, z);
      if constexpr (GATED) load8(Z + p.n, u);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float slope;
        const float d = v[i >> 2][i & 3], value = act_value_grad<C>(k, z[i >> 2][i & 3], &slope);
        if constexpr (GATED) {
          y[i >> 2][i & 3] = d * value;
          v[i >> 2][i & 3] = d * u[i >> 2][i & 3] * slope;
        } else {
          v[i >> 2][i & 3] = d * slope;
        }
      }
      if constexpr (GATED) store8(to + p.n, y);
    }
    store8(to, v);
  });
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
  p.splits = f.splits;
  p.part = f.splits > 1 ? static_cast<float*>(ws) : nullptr;
  p.act = s.act;
  p.f32 = c.f32;
  p.accumulate = c.accumulate;
  p.n = (int32_t)(direction == GROUPED_GRAD ? s.in : s.out);
  p.k = (int32_t)(direction == GROUPED_GRAD ? s.out : s.in);
  p.ldv = s.w_ld;
  if (direction == GROUPED_WGRAD) {
    p.ldv = c.b_ld;
    p.ld_out = s.w_ld;
  }
  const unsigned groups = (unsigned)f.workgroups;
  const auto rows = [&](auto tile, auto grad) {
    using T = decltype(tile);
    constexpr bool G = decltype(grad)::value;
    if (s.gated) hipLaunchKernelGGL((grouped_rows_kernel<T, G, true>), dim3(groups), dim3(T::THREADS), 0, stream, p);
    else hipLaunchKernelGGL((grouped_rows_kernel<T, G, false>), dim3(groups), dim3(T::THREADS), 0, stream, p);
  };
  const auto wgrad = [&](auto tile) {
    using T = decltype(tile);
    if (p.accumulate || p.part) hipLaunchKernelGGL((grouped_wgrad_kernel<T, WGRAD_ANY>), dim3(groups), dim3(T::THREADS), 0, stream, p);
    else if (p.f32) hipLaunchKernelGGL((grouped_wgrad_kernel<T, WGRAD_F32>), dim3(groups), dim3(T::THREADS), 0, stream, p);
    else hipLaunchKernelGGL((grouped_wgrad_kernel<T, WGRAD_BF16>), dim3(groups), dim3(T::THREADS), 0, stream, p);
  };
  const std::true_type yes;
  const std::false_type no;
  if (direction == GROUPED_WGRAD) {
    if (f.tile_n == 256) wgrad(ProductTile<256, 256, false, false, 2, 8, 4>{});
    else wgrad(ProductTile<128, 128, false, false, 2, 8, 2>{});
  } else if (direction == GROUPED_FORWARD) {
    if (f.tile_m == 256) rows(ProductTile<256, 256, true, true, 2, 8, 4, true>{}, no);
    else if (f.tile_m == 128) rows(ProductTile<128, 128, true, true, 2, 8, 2, true>{}, no);
    else rows(ProductTile<64, 128, true, true, 3, 8, 2, true>{}, no);
  } else {
    if (f.tile_m == 256) rows(ProductTile<256, 256, true, false, 2, 8, 4, true>{}, yes);
    else if (f.tile_m == 128) rows(ProductTile<128, 128, true, false, 2, 8, 2, true>{}, yes);
    else rows(ProductTile<64, 128, true, false, 3, 8, 2, true>{}, yes);
  }
  if (hipError_t e = hipGetLastError()) return e;
  if (f.splits == 1) return hipSuccess;
  const int64_t rows8 = direction == GROUPED_WGRAD ? (int64_t)p.experts * p.n : p.rows;
  const int64_t cols8 = direction == GROUPED_WGRAD ? p.k / 8 : direction == GROUPED_FORWARD && s.gated ? p.n / 16 : p.n / 8;
  const dim3 sums((unsigned)((rows8 * cols8 + 255) / 256));
  if (direction == GROUPED_WGRAD) hipLaunchKernelGGL((grouped_sum_kernel<GROUPED_WGRAD, false>), sums, dim3(256), 0, stream, p);
  else if (direction == GROUPED_FORWARD && s.gated) hipLaunchKernelGGL((grouped_sum_kernel<GROUPED_FORWARD, true>), sums, dim3(256), 0, stream, p);
  else if (direction == GROUPED_FORWARD) hipLaunchKernelGGL((grouped_sum_kernel<GROUPED_FORWARD, false>), sums, dim3(256), 0, stream, p);
  else if (s.gated) hipLaunchKernelGGL((grouped_sum_kernel<GROUPED_GRAD, true>), sums, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL((grouped_sum_kernel<GROUPED_GRAD, false>), sums, dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace ccl
