// Epilogues of ccl_gemm_fused and ccl_gemm_fused_grad on a tile of the
// product D = A B. Included by gemm_tiles.hpp inside its namespace.
//
// Forward:  Z = alpha D + bias, C = act(Z) + beta R; gated: the columns of D
//           alternate in groups of 16, gate and up, and C = act(Zg) Zu + beta R
//           has half as many. Z is kept in bf16 where asked for; C is formed
//           from the fp32 Z and rounded once.
// Backward: dZ = alpha D act'(Z); gated: D is the gradient of the half-width
//           C, dZg = alpha D Zu act'(Zg), dZu = alpha D act(Zg). The column
//           sums of the fp32 dZ (the bias gradient) are formed tile by tile
//           and added up in ascending row order by bias_reduce_kernel.
// Rows at and past `rows` come out as zeros; nothing of D, R or Z reaches them.
//
// What it adds to the product, us (product alone -> with it): SwiGLU with Z kept, 4096x1536x2048, 24.7 -> 27.3; dZ of a gated
// 4096x768x2048 15.7 -> 22.1 (25 MB of Z and dZ behind a K loop of 10 us); GELU with
// Z kept, 8192x28672x8192, 2596 -> 2690. Reading R and Z and storing wait on memory
// while the workgroup's matrix cores idle: short K takes tiles of which two share
// a CU (fused_form's rule).
//
// On 256x256 tiles the accumulators take half of the 256 registers, and the
// epilogue's values spill: 198 to 211 registers in the gradient kernels, nearly all
// behind the K loop, and 11 in the pipelined fp8 forward kernel, 16 of whose 20
// accesses lie in the K loop, where their waits drain its loads (4096x57344x8192
// gated 1543 us, 2.49 PFLOP/s; ccl_gemm on the same kind of tiles 2.95).

struct FusedEpi {
  const void* bias;         // per column of D (null: none)
  const uint16_t* R;        // residual, laid out as C (null: none)
  const uint16_t* Zin;      // backward: pre-activations, laid out as dZ (null: not needed)
  uint16_t* Zout;           // forward: pre-activations to keep (null: none)
  float* colsum;            // backward: [row blocks][columns of dZ] (null: none)
  OperandAddr z;            // addressing of Zin / Zout (GemmParams::c: of C / dZ)
  int64_t rows;             // valid rows
  int64_t part_rows;        // rows of a partition, M / Gr
  int64_t z_cols;           // columns of Z: N, or 2 N in the gated backward
  int32_t part_cols;        // columns of D in a partition, N / Gc
  int32_t act, gated, bias_f32;
  float beta;
};

struct FusedParams : GemmParams {
  FusedEpi e;
  LiveMap live;             // read where remap is 0
};

// The tile of this workgroup: its owner's (remap), or by the map over the tiles
// that have valid rows.
__device__ __forceinline__ bool tile_of_block_raw(const FusedParams& p, int32_t* pr, int32_t* pc, int32_t* ti,
                                                  int32_t* tj, int32_t* split) {
  *split = 0;
  if (p.remap) return map_tile(p.map, blockIdx.x, pr, pc, ti, tj, split);
  return live_tile(p.live, blockIdx.x, pr, pc, ti, tj);
}

__device__ __forceinline__ f32x4 bf16x4_to_f32(uint2 b) {
  return f32x4{__uint_as_float(b.x << 16), __uint_as_float(b.x & 0xffff0000u), __uint_as_float(b.y << 16),
               __uint_as_float(b.y & 0xffff0000u)};
}

__device__ __forceinline__ uint2 f32_to_bf16x4(f32x4 o) {
  // The compiler's conversion (v_cvt_pk_bf16_f32): nearest even, NaN kept.
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(uint2, __builtin_convertvector(o, bf16x4));
}

// Bias of four consecutive columns from column n of D.
__device__ __forceinline__ f32x4 bias4(const FusedEpi& e, int64_t n) {
  if (!e.bias) return f32x4{0.f, 0.f, 0.f, 0.f};
  if (e.bias_f32) return *reinterpret_cast<const f32x4*>(static_cast<const float*>(e.bias) + n);
  return bf16x4_to_f32(*reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(e.bias) + n));
}

// Gated column pairs: column n of the half-width matrix has its gate at
// wide_col(n) and its up at wide_col(n) + 16; n and n + 3 lie in one group.
__device__ __forceinline__ int wide_col(int n) { return ((n & ~15) << 1) | (n & 15); }

// ---------------------------------------------------------------------------
// The epilogue in the GEMM kernel itself (kernels with 16x16 MFMA tiles and 8
// waves). Lane l holds rows wm WM + 16 mt + l % 16 and columns wn WN + 16 nt +
// 4 (l / 16) .. + 3 of D in acc[mt][nt]; a gate and its up are acc[mt][2 i] and
// acc[mt][2 i + 1] of one lane, so the formulas stay in registers. Matrices
// cross between this order and whole 128-byte lines of memory through the
// stage buffers, idle after the K loop: what is read (R, Z) is copied in line
// by line and picked up 8 bytes a lane, the result replaces it in place, and
// lines are copied out.
// ---------------------------------------------------------------------------

// A bf16 matrix of ROWS x COLS in the two stage arrays, half of its rows in
// each, 16-byte chunks XORed with the row so that the 16 rows of one access
// fall in distinct banks: rows of 16 i chunks start in the same bank, of 8 i in
// two, of 4 i in four.
template <int ROWS, int COLS>
struct StagedTile {
  static constexpr int HALF = ROWS / 2, PITCH = COLS * 2, CPR = COLS / 8;
  static_assert(CPR % 4 == 0, "the swizzle is defined for rows of 4 i chunks");
  static constexpr int swizzle(int h) { return CPR % 16 == 0 ? h & 15 : CPR % 8 == 0 ? (h >> 1) & 7 : (h >> 2) & 3; }
  char *lo, *hi;
  __device__ __forceinline__ char* chunk(int r, int c) const {
    const int h = r < HALF ? r : r - HALF;
    return (r < HALF ? lo : hi) + h * PITCH + ((c ^ swizzle(h)) << 4);
  }
  // Four columns from column n (a multiple of 4) of row r.
  __device__ __forceinline__ uint2* at(int r, int n) const {
    return reinterpret_cast<uint2*>(chunk(r, n >> 3) + ((n >> 2) & 1) * 8);
  }
};

// Every LDS access of the workgroup before this is done after it.
__device__ __forceinline__ void staged_barrier() {
  __builtin_amdgcn_s_waitcnt(waitcnt_imm(63, 0));
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Staged row r is row `row(r)` of the matrix at m (leading dimension ld).
template <int ROWS, int COLS, int THREADS, typename Row>
__device__ __forceinline__ void copy_in(const StagedTile<ROWS, COLS>& t, const uint16_t* m, int32_t ld, int tid, Row&& row) {
  constexpr int CPR = COLS / 8, N = ROWS * CPR / THREADS;
  static_assert(ROWS * CPR % THREADS == 0, "whole accesses");
  // loads in flight per thread
  constexpr int B = N <= 8 ? N : N % 8 == 0 ? 8 : N % 6 == 0 ? 6 : N % 5 == 0 ? 5 : 1;
  static_assert(N % B == 0 && B > 1, "whole batches");
  for (int i = 0; i < N; i += B) {
    uint4 v[B];
#pragma unroll
    for (int j = 0; j < B; ++j) {
      const int at = (i + j) * THREADS + tid;
      v[j] = *reinterpret_cast<const uint4*>(m + (int64_t)row(at / CPR) * ld + at % CPR * 8);
    }
#pragma unroll
    for (int j = 0; j < B; ++j) {
      const int at = (i + j) * THREADS + tid;
      *reinterpret_cast<uint4*>(t.chunk(at / CPR, at % CPR)) = v[j];
    }
  }
}

template <int ROWS, int COLS, int THREADS, typename Row>
__device__ __forceinline__ void copy_out(const StagedTile<ROWS, COLS>& t, uint16_t* m, int32_t ld, int32_t nt, int tid,
                                         Row&& row) {
  constexpr int CPR = COLS / 8, N = ROWS * CPR / THREADS;
  choose_nt(nt, [&](auto past) __attribute__((always_inline)) {
#pragma unroll 4
    for (int i = 0; i < N; ++i) {
      const int at = i * THREADS + tid;
      const i32x4 v = *reinterpret_cast<const i32x4*>(t.chunk(at / CPR, at % CPR));
      i32x4* dst = reinterpret_cast<i32x4*>(m + (int64_t)row(at / CPR) * ld + at % CPR * 8);
      if constexpr (decltype(past)::value) __builtin_nontemporal_store(v, dst);
      else *dst = v;
    }
  });
}

template <int COLS, int THREADS>
__device__ __forceinline__ void zero_rows(uint16_t* m, int32_t ld, int rows, int tid) {
  constexpr int CPR = COLS / 8;
  for (int at = tid; at < rows * CPR; at += THREADS)
    *reinterpret_cast<uint4*>(m + (int64_t)(at / CPR) * ld + at % CPR * 8) = make_uint4(0, 0, 0, 0);
}

// Corners of a tile (or of its 2 BN or BN / 2 columns) in a matrix.
template <int BM>
__device__ __forceinline__ int64_t tile_corner(const OperandAddr& o, int32_t pr, int32_t pc, int32_t ti, int64_t col) {
  return pr * o.part + pc * o.slice + (int64_t)(ti * BM) * o.ld + col;
}

// A tile wholly past the valid rows: zeros, and no column sums or partials (the
// reduces do not read them; with partials, theirs writes the zeros). Whether it
// was one.
template <int BM, int BN, int THREADS, bool GRAD>
__device__ __forceinline__ bool dead_tile(const FusedParams& p, int32_t pr, int32_t pc, int32_t ti, int32_t tj) {
  const FusedEpi& e = p.e;
  if (pr * e.part_rows + (int64_t)ti * BM < e.rows) return false;
  if (p.ws) return true;
  const int tid = threadIdx.x;
  uint16_t* C = static_cast<uint16_t*>(p.C);
  const auto zero = [&](uint16_t* m, const OperandAddr& o, auto cols) {
    constexpr int W = decltype(cols)::value;
    zero_rows<W, THREADS>(m + tile_corner<BM>(o, pr, pc, ti, (int64_t)tj * W), o.ld, BM, tid);
  };
  if (!e.gated) zero(C, p.c, std::integral_constant<int, BN>{});
  else zero(C, p.c, std::integral_constant<int, GRAD ? 2 * BN : BN / 2>{});
  if (!GRAD && e.Zout) zero(e.Zout, e.z, std::integral_constant<int, BN>{});
  return true;
}

template <int BM, int BN, int NW, int TM, int TN, int WM, int WN>
__device__ __forceinline__ void fused_forward(const FusedParams& p, f32x4 (&acc)[TM][TN], char* lo, char* hi,
                                              int32_t pr, int32_t pc, int32_t ti, int32_t tj, int wm, int wn, int tid) {
  const FusedEpi& e = p.e;
  constexpr int THREADS = 64 * NW;
  const int lane = tid & 63;
  const int r0 = wm * WM + (lane & 15), n0 = wn * WN + 4 * (lane >> 4);
  const int64_t left = e.rows - (pr * e.part_rows + (int64_t)ti * BM);   // valid rows from the tile's first on
  const auto same = [](int r) { return r; };
  const f32x4 zero{0.f, 0.f, 0.f, 0.f};
  // Z, in place of D
#pragma unroll
  for (int nt = 0; nt < TN; ++nt) {
    const f32x4 b = bias4(e, pc * (int64_t)e.part_cols + tj * BN + n0 + 16 * nt);
#pragma unroll
    for (int mt = 0; mt < TM; ++mt) {
      const bool live = r0 + 16 * mt < left;
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[mt][nt][j] = live ? __builtin_fmaf(p.alpha, acc[mt][nt][j], b[j]) : 0.f;
    }
  }
  if (e.Zout) {
    const StagedTile<BM, BN> t{lo, hi};
#pragma unroll
    for (int mt = 0; mt < TM; ++mt)
#pragma unroll
      for (int nt = 0; nt < TN; ++nt) *t.at(r0 + 16 * mt, n0 + 16 * nt) = f32_to_bf16x4(acc[mt][nt]);
    staged_barrier();
    copy_out<BM, BN, THREADS>(t, e.Zout + tile_corner<BM>(e.z, pr, pc, ti, tj * BN), e.z.ld, p.c_nt, tid, same);
    staged_barrier();
  }
  const ActCoef k = act_coef(e.act);
  const auto finish = [&](auto gated) __attribute__((always_inline)) {
    constexpr bool GATED = decltype(gated)::value;
    constexpr int W = GATED ? BN / 2 : BN;
    const StagedTile<BM, W> t{lo, hi};
    const int64_t corner = tile_corner<BM>(p.c, pr, pc, ti, (int64_t)tj * W);
    if (e.R) {
      copy_in<BM, W, THREADS>(t, e.R + corner, p.c.ld, tid, same);
      staged_barrier();
    }
    with_act(e.act, [&](auto cls) __attribute__((always_inline)) {
#pragma unroll
      for (int mt = 0; mt < TM; ++mt) {
        const bool live = r0 + 16 * mt < left;
#pragma unroll
        for (int nt = 0; nt < TN; nt += GATED ? 2 : 1) {
          uint2* at = t.at(r0 + 16 * mt, GATED ? wn * (WN / 2) + 4 * (lane >> 4) + 8 * nt : n0 + 16 * nt);
          f32x4 o;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            o[j] = act_value<decltype(cls)::value>(k, acc[mt][nt][j]);
            if constexpr (GATED) o[j] *= acc[mt][nt + 1][j];
          }
          if (e.R) {
            const f32x4 r = bf16x4_to_f32(*at);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = __builtin_fmaf(e.beta, r[j], o[j]);
          }
          *at = f32_to_bf16x4(live ? o : zero);
        }
      }
    });
    staged_barrier();
    copy_out<BM, W, THREADS>(t, static_cast<uint16_t*>(p.C) + corner, p.c.ld, p.c_nt, tid, same);
  };
  // A wave with an odd number of 16-column tiles splits a pair: those kernels are
  // not launched on gated products.
  if constexpr (TN % 2 == 0) {
    if (e.gated) {
      finish(std::true_type{});
      return;
    }
  }
  finish(std::false_type{});
}

template <int BM, int BN, int NW, int TM, int TN, int WM, int WN>
__device__ __forceinline__ void fused_backward(const FusedParams& p, const f32x4 (&acc)[TM][TN], char* lo, char* hi,
                                               int32_t pr, int32_t pc, int32_t ti, int32_t tj, int wm, int wn, int tid) {
  const FusedEpi& e = p.e;
  constexpr int THREADS = 64 * NW;
  const int lane = tid & 63;
  const int64_t left = e.rows - (pr * e.part_rows + (int64_t)ti * BM);
  const ActCoef k = act_coef(e.act);
  const f32x4 zero{0.f, 0.f, 0.f, 0.f};
  const auto finish = [&](auto gated) __attribute__((always_inline)) {
    constexpr bool GATED = decltype(gated)::value;
    // A gated Z and dZ have 2 BN columns: two passes of half of every wave's rows.
    constexpr int PASSES = GATED ? 2 : 1;
    constexpr int W = GATED ? 2 * BN : BN, PM = WM / PASSES;
    const StagedTile<BM / PASSES, W> t{lo, hi};
    const int64_t corner = tile_corner<BM>(p.c, pr, pc, ti, (int64_t)tj * W);
    f32x4 sums[TN][PASSES];
#pragma unroll
    for (int nt = 0; nt < TN; ++nt)
#pragma unroll
      for (int h = 0; h < PASSES; ++h) sums[nt][h] = zero;
#pragma unroll
    for (int ps = 0; ps < PASSES; ++ps) {
      const auto row = [&](int r) { return r / PM * WM + ps * PM + r % PM; };
      if (ps) staged_barrier();               // the pass before has been copied out
      if (e.Zin) {
        copy_in<BM / PASSES, W, THREADS>(t, e.Zin + corner, p.c.ld, tid, row);
        staged_barrier();
      }
      with_act(e.act, [&](auto cls) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < TM / PASSES; ++m) {
          const int mt = ps * (TM / PASSES) + m;
          const bool live = wm * WM + 16 * mt + (lane & 15) < left;
          const int r = wm * PM + 16 * m + (lane & 15);
#pragma unroll
          for (int nt = 0; nt < TN; ++nt) {
            const int n = wn * (W / (BN / WN)) + 4 * (lane >> 4) + (GATED ? 32 : 16) * nt;
            const f32x4 z = e.Zin ? bf16x4_to_f32(*t.at(r, n)) : zero;
            f32x4 zu = zero, u = zero, g;
            if constexpr (GATED) zu = bf16x4_to_f32(*t.at(r, n + 16));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float d = p.alpha * acc[mt][nt][j];
              float grad;
              const float value = act_value_grad<decltype(cls)::value>(k, z[j], &grad);
              g[j] = d * grad;
              if constexpr (GATED) {
                g[j] *= zu[j];
                u[j] = d * value;
              }
            }
            g = live ? g : zero;
            *t.at(r, n) = f32_to_bf16x4(g);
            sums[nt][0] += g;
            if constexpr (GATED) {
              u = live ? u : zero;
              *t.at(r, n + 16) = f32_to_bf16x4(u);
              sums[nt][PASSES - 1] += u;
            }
          }
        }
      });
      staged_barrier();
      copy_out<BM / PASSES, W, THREADS>(t, static_cast<uint16_t*>(p.C) + corner, p.c.ld, p.c_nt, tid, row);
    }
    if (!e.colsum) return;
    // Over the 16 rows of a lane group, then over the rows of waves in order.
    staged_barrier();
    float* part = reinterpret_cast<float*>(lo);       // [BM / WM][W]
#pragma unroll
    for (int nt = 0; nt < TN; ++nt)
#pragma unroll
      for (int h = 0; h < PASSES; ++h) {
        f32x4 v = sums[nt][h];
#pragma unroll
        for (int x = 1; x < 16; x <<= 1)
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] += __shfl_xor(v[j], x);
        const int n = wn * (W / (BN / WN)) + 4 * (lane >> 4) + (GATED ? 32 : 16) * nt + 16 * h;
        if ((lane & 15) == 0) *reinterpret_cast<f32x4*>(part + wm * W + n) = v;
      }
    staged_barrier();
    float* to = e.colsum + (pr * e.part_rows + (int64_t)ti * BM) / BM * e.z_cols +
                (W / BN) * pc * (int64_t)e.part_cols + (int64_t)tj * W;
    for (int n = tid; n < W; n += THREADS) {
      float v = part[n];
#pragma unroll
      for (int w = 1; w < BM / WM; ++w) v += part[w * W + n];
      to[n] = v;
    }
  };
  if (e.gated) finish(std::true_type{});
  else finish(std::false_type{});
}

// The parameters of a kernel with one direction's epilogue.
template <bool GRAD>
struct FusedTileParams : FusedParams {
  static constexpr bool kGrad = GRAD;
};

template <int BM, int BN, int NW, int TM, int TN, int WM, int WN, bool GRAD>
__device__ __forceinline__ void fused_epilogue(const FusedTileParams<GRAD>& p, f32x4 (&acc)[TM][TN], char* lo, char* hi,
                                               int32_t pr, int32_t pc, int32_t ti, int32_t tj, int wm, int wn, int tid) {
  // No wave reads the stage buffers any more and no load into them is in
  // flight (the direct-to-LDS loads of the last steps included).
  __builtin_amdgcn_s_waitcnt(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  if constexpr (GRAD) fused_backward<BM, BN, NW, TM, TN, WM, WN>(p, acc, lo, hi, pr, pc, ti, tj, wm, wn, tid);
  else fused_forward<BM, BN, NW, TM, TN, WM, WN>(p, acc, lo, hi, pr, pc, ti, tj, wm, wn, tid);
}
