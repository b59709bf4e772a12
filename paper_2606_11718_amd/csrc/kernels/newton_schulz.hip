// Orthogonalised updates (ccl_orthogonalize): Newton-Schulz steps of an odd
// quintic on a batch of matrices,
//   X = G / (|G|_F + eps), transposed if tall (p = min side, q = max side)
//   S = X X^T;  B = b S + c S S + s I;  X <- (a - s) X + B X       (each step;
//   s = -(b + c), which leaves B near 0 where S is near I)
// The three products of a step are matrix products with an addend, out = alpha
// U V' + beta D, on the matrix cores. S and B are symmetric: only the tiles on
// and below the diagonal are computed, each stored twice, which halves two of
// the three products (p^2 q + p^3 + 2 p^2 q operations a step against 2 p^2 q +
// 2 p^3 + 2 p^2 q).
//
// X, S and B are held in fp16 (the operands of v_mfma_f32_16x16x32_f16) times
// 2^13, with fp32 sums. With the default coefficients the singular values of X
// stay below 1.3, so every element of X, S and B is below 3 and 2^13 of it
// below fp16's 65504, while 2^13 keeps elements down to 2^-27 at full
// precision (those of a first X of 8192 x 28672 are around 2^-14). The 11 bits
// leave the result 0.9e-3 (wide) to 1.4e-3 (square) from the 64-bit one; with few
// singular values the roundings average out less (worst of 128 matrices: 1.7e-3 of
// 100 x 4200 and 64 x 64, 2.3e-3 of 32 x 32, 4.6e-3 of 16 x 16). bf16 iterates, with 8
// bits: 1e-2.
//
// Sides are padded to multiples of 128 with zeros, which the steps keep in X and S;
// on B's padded diagonal lies s, which meets X's zeros only.
//
// Measured, us a call of five steps (PFLOP/s of the operations above): 768x2048
// 134 (0.15: 17 dependent launches of 4 to 9), 16 of 2048x1536 1772 (0.82: 128x128
// tiles in the symmetric products, three rounds of 256x256 in the third), 8192x28672
// 24100 to 24900 (1.27 to 1.31: the matrix cores at the power limit).
#include "gemm_tiles.hpp"

namespace ccl {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) f16x8 lds_f16x8;

constexpr float kScale = 8192.f;      // of the stored X, S and B

struct NsParams {
  const uint16_t* U;        // M x K, K contiguous
  const uint16_t* V;        // NT: N x K, K contiguous; else K x N
  const uint16_t* D;        // addend, laid out as out (null: none)
  uint16_t* out;            // fp16 M x N
  uint16_t* O;              // the last product: bf16 result instead of out (else null)
  float* part;              // fp32 tiles of the ranges of the split ones, in fragment order
  int64_t u_stride, v_stride, out_stride, o_stride;   // elements between matrices (D: out's)
  int64_t o_ld;
  int32_t M, N, K;          // padded
  int32_t ldu, ldv, ld_out;
  int32_t o_rows, o_cols;   // of the result; o_trans: it is the transpose of the product
  int32_t o_trans;
  int32_t tiles_m, tiles_n; // per matrix; symmetric: tiles_m (tiles_m + 1) / 2 tiles
  int32_t tiles, total;     // per matrix, of the launch
  int32_t group;
  int32_t whole;            // tiles computed by one workgroup each (a multiple of 8, or all)
  int32_t splits, ksplit;   // the other tiles' K ranges, of ksplit steps
  int32_t whole_xcd, split_xcd;   // workgroups of each kind per XCD
  float alpha, beta;
  float diag;               // added on the diagonal of a symmetric out
};

// 8 waves, 2 x 4. (64x64 in 2 x 2 waves reads a third less of LDS a step and took
// 6 to 9 % longer.)
template <int BM, int BN, bool NT, int NS_>
struct NsTile {
  static constexpr int WGN = 4, NW = 8, THREADS = 512;
  static constexpr int WM = BM / 2, WN = BN / WGN;
  static constexpr int TM = WM / 16, TN = WN / 16;
  static constexpr int U_BYTES = BM * 128, V_BYTES = BN * 128;   // a stage of 64 K
  static constexpr int NU = U_BYTES / (1024 * NW), NV = V_BYTES / (1024 * NW), NL = NU + NV;
  static constexpr int CPR_V = BN / 8, RPI_V = 64 / CPR_V;       // 16-byte chunks and rows of a load (not NT)
  static_assert(BM * BN / 8 % THREADS == 0, "whole copies");
  static constexpr int NS = NS_;
  // With two stage buffers a step's loads go out behind its barrier, into the
  // buffer it has just read; otherwise NS - 1 stages ahead of it.
  static constexpr bool kLate = NS == 2;
  static constexpr int AHEAD = kLate ? 2 : NS - 1;
  static_assert(NS == 2 || NS == 4, "the waits of a step are written for these");
  static_assert(NU >= 1 && NV >= 1 && NU <= 4 && NV <= 4, "a run of loads shares one M0");
  static_assert((BM / 2) * BN * 2 <= NS * U_BYTES && (BM / 2) * BN * 2 <= NS * V_BYTES, "the tile is staged in both");
};

// Tile t of a matrix: tile rows in groups, column by column.
template <bool SYM>
__device__ __forceinline__ void ns_tile(const NsParams& p, int32_t t, int32_t* ti, int32_t* tj) {
  const int32_t G = p.group;
  if constexpr (SYM) {
    // rows G r .. G r + G - 1 have G r (G r + 1) / 2 tiles before them
    int32_t r = 0;
    while (G * (r + 1) < p.tiles_m && (G * (r + 1)) * (G * (r + 1) + 1) / 2 <= t) ++r;
    const int32_t first = G * r, h = min(G, p.tiles_m - first);
    int32_t w = t - first * (first + 1) / 2;
    if (w < h * (first + 1)) {          // columns that every row of the group has
      *tj = w / h;
      *ti = first + w - *tj * h;
    } else {                            // the group's own triangle, below the diagonal's first column
      w -= h * (first + 1);
      int32_t j = first + 1;
      while (w >= h - (j - first)) {
        w -= h - (j - first);
        ++j;
      }
      *tj = j;
      *ti = j + w;
    }
  } else {
    const int32_t per = G * p.tiles_n, r = t / per, first = r * G, h = min(G, p.tiles_m - first);
    const int32_t w = t - r * per;
    *tj = w / h;
    *ti = first + w - *tj * h;
  }
}

// Workgroup -> matrix, tile and K steps [*k0, *k1). The tiles of all matrices
// are numbered matrix by matrix and each XCD (workgroup mod 8) takes a
// contiguous range of them, so that what is resident on one XCD together shares
// operands in its L2. The tiles past p.whole are cut along K: with them, the
// last round of workgroups fills the CUs (*part: where the range's partial
// tile goes, else -1).
template <bool SYM>
__device__ __forceinline__ bool ns_work(const NsParams& p, int32_t* mat, int32_t* ti, int32_t* tj, int32_t* k0,
                                        int32_t* k1, int32_t* part) {
  const int32_t xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
  int32_t id;
  if (slot < p.whole_xcd) {
    id = xcd * p.whole_xcd + slot;
    if (id >= p.whole) return false;
    *k0 = 0;
    *k1 = p.K / 64;
    *part = -1;
  } else {
    const int32_t v = xcd * p.split_xcd + slot - p.whole_xcd;
    if (v >= (p.total - p.whole) * p.splits) return false;
    const int32_t tile = v / p.splits, range = v - tile * p.splits;
    id = p.whole + tile;
    *k0 = __builtin_amdgcn_readfirstlane(range * p.ksplit);
    *k1 = __builtin_amdgcn_readfirstlane(min(p.K / 64, range * p.ksplit + p.ksplit));
    *part = __builtin_amdgcn_readfirstlane(v);
  }
  const int32_t m = id / p.tiles;
  int32_t i, j;
  ns_tile<SYM>(p, id - m * p.tiles, &i, &j);
  *mat = __builtin_amdgcn_readfirstlane(m);
  *ti = __builtin_amdgcn_readfirstlane(i);
  *tj = __builtin_amdgcn_readfirstlane(j);
  return true;
}

// Eight values to row r, columns c .. c + 7 of a matrix with `cols` columns.
__device__ __forceinline__ void store8(uint16_t* m, int64_t ld, int r, int c, int cols, uint4 v) {
  uint16_t* dst = m + r * ld + c;
  if (c + 8 <= cols && (reinterpret_cast<uintptr_t>(dst) & 15) == 0) {
    *reinterpret_cast<uint4*>(dst) = v;
    return;
  }
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (c + j < cols) dst[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
}

// The staged tile to rows r0 .. and columns c0 .. of a rows x cols matrix.
template <int BM, int BN, int THREADS>
__device__ __forceinline__ void ns_copy_out(const StagedTile<BM, BN>& t, uint16_t* m, int64_t ld, int r0, int c0,
                                            int rows, int cols, int tid) {
  constexpr int CPR = BN / 8;
#pragma unroll 4
  for (int i = 0; i < BM * CPR / THREADS; ++i) {
    const int at = i * THREADS + tid, r = at / CPR, c = at % CPR;
    const uint4 v = *reinterpret_cast<const uint4*>(t.chunk(r, c));
    if (r0 + r < rows && c0 + 8 * c < cols) store8(m, ld, r0 + r, c0 + 8 * c, cols, v);
  }
}

// Its transpose. ds_read_b64_tr_b16 hands lane l of 16 column l of the 4 x 16
// block that its 16 lanes read (lane s: row s / 4, columns 4 (s % 4) .. + 3):
// two of them are eight consecutive rows of one column.
template <int BM, int BN, int NW>
__device__ __forceinline__ void ns_copy_out_trans(const StagedTile<BM, BN>& t, uint16_t* m, int64_t ld, int r0, int c0,
                                                  int rows, int cols, int wave, int lane) {
  const int g = lane >> 4, s = lane & 15;
  constexpr int UNITS = (BM / 32) * (BN / 16) / NW;
#pragma unroll 2
  for (int i = 0; i < UNITS; ++i) {
    const int u = wave * UNITS + i;
    const int row = (u % (BM / 32)) * 32 + 8 * g, col = u / (BM / 32) * 16;
    const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(char*)t.at(row + (s >> 2), col + 4 * (s & 3)));
    const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(char*)t.at(row + 4 + (s >> 2), col + 4 * (s & 3)));
    const uint2 x = __builtin_bit_cast(uint2, a), y = __builtin_bit_cast(uint2, b);
    if (r0 + col + s < rows && c0 + row < cols) store8(m, ld, r0 + col + s, c0 + row, cols, make_uint4(x.x, x.y, y.x, y.y));
  }
}

// D's ROWS x COLS from row r0, column c0, through registers into the staged
// tile. (Accumulators that started from D instead, loaded in their own order with
// the first stages, took 1 to 5 % longer: 32-byte pieces.)
template <int ROWS, int COLS, int THREADS>
struct NsAddend {
  static constexpr int CPR = COLS / 8, N = ROWS * CPR / THREADS, B = N < 8 ? N : 8;
  uint4 v[B];
  __device__ __forceinline__ void load(const NsParams& p, int mat, int r0, int c0, int i, int tid) {
    const uint16_t* d = p.D + mat * p.out_stride;
#pragma unroll
    for (int j = 0; j < B; ++j) {
      const int at = (i + j) * THREADS + tid, r = r0 + at / CPR, c = c0 + at % CPR * 8;
      v[j] = make_uint4(0, 0, 0, 0);
      if (r < p.M && c < p.N) v[j] = *reinterpret_cast<const uint4*>(d + (int64_t)r * p.ld_out + c);
    }
  }
  __device__ __forceinline__ void put(const StagedTile<ROWS, COLS>& t, int i, int tid) const {
#pragma unroll
    for (int j = 0; j < B; ++j) {
      const int at = (i + j) * THREADS + tid;
      *reinterpret_cast<uint4*>(t.chunk(at / CPR, at % CPR)) = v[j];
    }
  }
};

template <int ROWS, int COLS, int THREADS>
__device__ __forceinline__ void ns_copy_in(const NsParams& p, const StagedTile<ROWS, COLS>& t, int mat, int r0, int c0,
                                           int tid) {
  using A = NsAddend<ROWS, COLS, THREADS>;
  for (int i = 0; i < A::N; i += A::B) {
    A a;
    a.load(p, mat, r0, c0, i, tid);
    a.put(t, i, tid);
  }
}

// alpha acc + beta D + diag I on four staged values of row r, columns c .. c + 3,
// in place.
template <bool SYM>
__device__ __forceinline__ void ns_combine(const NsParams& p, uint2* at, f32x4 acc, int r, int c) {
  f32x4 o = acc * p.alpha;
  if constexpr (SYM) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (r == c + j) o[j] += p.diag;
  }
  if (p.D) {
    const f16x4 d = __builtin_bit_cast(f16x4, *at);
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = __builtin_fmaf(p.beta, (float)d[j], o[j]);
  }
  *at = p.O ? f32_to_bf16x4(o) : __builtin_bit_cast(uint2, __builtin_convertvector(o, f16x4));
}

// The staged tile (corner r0, c0) to where it goes: the result, or out, and off
// the diagonal of a symmetric out to its mirror image.
template <int ROWS, int COLS, bool SYM>
__device__ __forceinline__ void ns_store(const NsParams& p, const StagedTile<ROWS, COLS>& t, int mat, int r0, int c0,
                                         bool off_diagonal, int tid) {
  const int wave = tid >> 6, lane = tid & 63;
  if (p.O) {
    uint16_t* O = p.O + mat * p.o_stride;
    if (p.o_trans) ns_copy_out_trans<ROWS, COLS, 8>(t, O, p.o_ld, c0, r0, p.o_rows, p.o_cols, wave, lane);
    else ns_copy_out<ROWS, COLS, 512>(t, O, p.o_ld, r0, c0, p.o_rows, p.o_cols, tid);
    return;
  }
  uint16_t* out = p.out + mat * p.out_stride;
  ns_copy_out<ROWS, COLS, 512>(t, out, p.ld_out, r0, c0, p.M, p.N, tid);
  if (SYM && off_diagonal) ns_copy_out_trans<ROWS, COLS, 8>(t, out, p.ld_out, c0, r0, p.N, p.M, wave, lane);
}

// out = alpha U V' + beta D. The K loop is that of the GEMM's 64-K tiles: a
// stage's two halves of 32 K around one barrier, the next half's fragments read
// behind the MFMAs. U rows are 128 bytes with chunk c of row r at c ^
// swz_a64(r), V's the same (NT) or 64 rows of BN with the transposing reads.
// The symmetric products have K contiguous in both operands (NT).
template <int BM, int BN, bool SYM, int NS>
__global__ void __launch_bounds__(512, NS * (BM + BN) * 128 <= 80 * 1024 ? 4 : 2) ns_product_kernel(NsParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr bool NT = SYM;
  using T = NsTile<BM, BN, NT, NS>;
  __shared__ __attribute__((aligned(1024))) char smU[NS][T::U_BYTES];
  __shared__ __attribute__((aligned(1024))) char smV[NS][T::V_BYTES];
  int32_t mat, ti, tj, k0, k1, part;
  if (!ns_work<SYM>(p, &mat, &ti, &tj, &k0, &k1, &part)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / T::WGN, wn = wave % T::WGN;
  const int32_t ksteps = k1 - k0;

  // Per-lane byte offsets of the loads, minus the instruction offset of load i
  // of its run (rows are at least 128 elements: never negative).
  uint32_t u_voff[T::NU], v_voff[T::NV];
#pragma unroll
  for (int i = 0; i < T::NU; ++i) {
    const int row = 8 * (wave * T::NU + i) + (lane >> 3);
    u_voff[i] = (uint32_t)(row * p.ldu + ((lane & 7) ^ swz_a64(row)) * 8) * 2u - 1024u * i;
  }
#pragma unroll
  for (int i = 0; i < T::NV; ++i) {
    if constexpr (NT) {
      const int row = 8 * (wave * T::NV + i) + (lane >> 3);
      v_voff[i] = (uint32_t)(row * p.ldv + ((lane & 7) ^ swz_a64(row)) * 8) * 2u - 1024u * i;
    } else {
      const int row = T::RPI_V * (wave * T::NV + i) + lane / T::CPR_V;
      v_voff[i] = (uint32_t)(row * p.ldv + ((lane % T::CPR_V) ^ swz_b(row)) * 8) * 2u - 1024u * i;
    }
  }
  // Rows past the matrix read as zeros; columns past it (not NT) as the next
  // row's, which reach only columns that are not stored.
  const uint16_t* u0 = p.U + mat * p.u_stride + (int64_t)(ti * BM) * p.ldu;
  const uint16_t* v0 = p.V + mat * p.v_stride + (NT ? (int64_t)(tj * BN) * p.ldv : tj * BN);
  i32x4 u_desc = buffer_rsrc(u0, (int32_t)((int64_t)min(BM, p.M - ti * BM) * p.ldu * 2));
  i32x4 v_desc = buffer_rsrc(v0, NT ? (int32_t)((int64_t)min(BN, p.N - tj * BN) * p.ldv * 2)
                                    : (int32_t)(((int64_t)p.K * p.ldv - tj * BN) * 2));
  const uint32_t v_adv = NT ? 128u : (uint32_t)p.ldv * 128u;

  int32_t u_rd[2], v_rd[NT ? 1 : T::TN][2];
  {
    const int row = wm * T::WM + (lane & 15);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) u_rd[kk] = row * 128 + (((4 * kk + (lane >> 4)) ^ swz_a64(row)) * 16);
  }
  if constexpr (NT) {
    const int row = wn * T::WN + (lane & 15);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) v_rd[0][kk] = row * 128 + (((4 * kk + (lane >> 4)) ^ swz_a64(row)) * 16);
  } else {
    const int g = lane >> 4, s = lane & 15;
#pragma unroll
    for (int nt = 0; nt < T::TN; ++nt)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int krow = 8 * g + 4 * r + (s >> 2), col = wn * T::WN + nt * 16 + 4 * (s & 3);
        v_rd[nt][r] = krow * (BN * 2) + (((col >> 3) ^ swz_b(krow)) * 16) + ((col >> 2) & 1) * 8;
      }
  }

  auto load_one = [&](int32_t s, int i) __attribute__((always_inline)) {
    char* su = smU[0] + (s % NS) * T::U_BYTES;
    char* sv = smV[0] + (s % NS) * T::V_BYTES;
    if (i < T::NU) lds_dma16_run<false>(u_desc, u_voff[i], (uint32_t)(k0 + s) * 128u, su + (wave * T::NU + i) * 1024, i);
    else lds_dma16_run<false>(v_desc, v_voff[i - T::NU], (uint32_t)(k0 + s) * v_adv, sv + (wave * T::NV + i - T::NU) * 1024, i - T::NU);
  };
  // Loads past the last stage must not touch memory, but keep the count.
  auto end_loads = [&](int32_t s) __attribute__((always_inline)) {
    if (s >= ksteps) u_desc[2] = v_desc[2] = 0;
  };

  f16x8 fu0[T::TM], fu1[T::TM];
  i16x4 fv0[T::TN][2], fv1[T::TN][2];
  auto read_u = [&](const char* su, f16x8 (&f)[T::TM], int kk, int mt) __attribute__((always_inline)) {
    f[mt] = *(const lds_f16x8*)(su + u_rd[kk] + mt * 16 * 128);
  };
  constexpr int kVReads = NT ? T::TN : 2 * T::TN;
  auto read_v = [&](const char* sv, i16x4 (&f)[T::TN][2], int kk, int i) __attribute__((always_inline)) {
    if constexpr (NT) {
      const f16x8 v = *(const lds_f16x8*)(sv + v_rd[0][kk] + i * 16 * 128);
      typedef short i16x8 __attribute__((ext_vector_type(8)));
      const i16x8 w = __builtin_bit_cast(i16x8, v);
      f[i][0] = __builtin_shufflevector(w, w, 0, 1, 2, 3);
      f[i][1] = __builtin_shufflevector(w, w, 4, 5, 6, 7);
    } else {
      f[i >> 1][i & 1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(sv + v_rd[i >> 1][i & 1] + kk * 32 * BN * 2));
    }
  };

  // D of the 64-row tiles is loaded ahead of the stages, so that the epilogue
  // does not wait for it (17 launches of 128x128: 68.0 -> 67.5 us; of the 128x128
  // tiles, whose registers it takes, 3 of 1000x2000 242 -> 247).
  using Addend = NsAddend<BM, BN, T::THREADS>;
  constexpr bool kEarly = Addend::N == Addend::B && Addend::N <= 2;
  Addend early;
  if (kEarly && p.D && part < 0) early.load(p, mat, ti * BM, tj * BN, 0, tid);

  f32x4 acc[T::TM][T::TN];
#pragma unroll
  for (int i = 0; i < T::TM; ++i)
#pragma unroll
    for (int j = 0; j < T::TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto mfma_one = [&](const f16x8 (&fu)[T::TM], const i16x4 (&fv)[T::TN][2], int mt, int nt) __attribute__((always_inline)) {
    const f16x8 v = __builtin_bit_cast(f16x8, __builtin_shufflevector(fv[nt][0], fv[nt][1], 0, 1, 2, 3, 4, 5, 6, 7));
    acc[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, fu[mt], acc[mt][nt], 0, 0, 0);
  };
  auto stage_barrier = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(waitcnt_imm((NS - 2) * T::NL, 0));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  // Step s in stage buffer ph = s % NS; on entry fu0 / fv0 hold its first half.
  auto step = [&](int ph, int32_t s) __attribute__((always_inline)) {
    const char *su = smU[ph], *sv = smV[ph], *nu = smU[(ph + 1) % NS], *nv = smV[(ph + 1) % NS];
    constexpr int kMfma = T::TM * T::TN, kReads = T::TM + kVReads, kOps1 = kReads + (T::kLate ? 0 : T::NL);
    constexpr int kAll1 = kMfma > kOps1 ? kMfma : kOps1;
    end_loads(s + T::AHEAD);
    const auto load = [&](int i) __attribute__((always_inline)) {
      const int at = (ph + T::AHEAD) % NS;
      if (i < T::NU) lds_dma16_run<false>(u_desc, u_voff[i], (uint32_t)(k0 + s + T::AHEAD) * 128u, smU[at] + (wave * T::NU + i) * 1024, i);
      else lds_dma16_run<false>(v_desc, v_voff[i - T::NU], (uint32_t)(k0 + s + T::AHEAD) * v_adv, smV[at] + (wave * T::NV + i - T::NU) * 1024, i - T::NU);
    };
#pragma unroll
    for (int i = 0; i < kAll1; ++i) {
      if (i < kMfma) mfma_one(fu0, fv0, i / T::TN, i % T::TN);
      if (i < T::TM) read_u(su, fu1, 1, i);
      else if (i < kReads) read_v(sv, fv1, 1, i - T::TM);
      else if (i < kOps1) load(i - kReads);
      __builtin_amdgcn_sched_barrier(0);
    }
    stage_barrier();
    constexpr int kOps2 = kReads > T::NL ? kReads : T::NL;
    constexpr int kAll2 = kMfma > kOps2 ? kMfma : kOps2;
#pragma unroll
    for (int i = 0; i < kAll2; ++i) {
      if (i < kMfma) mfma_one(fu1, fv1, i / T::TN, i % T::TN);
      if (i < T::TM) read_u(nu, fu0, 0, i);
      else if (i < kReads) read_v(nv, fv0, 0, i - T::TM);
      if (T::kLate && i < T::NL) load(i);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

#pragma unroll
  for (int j = 0; j < T::AHEAD; ++j) {
    end_loads(j);
#pragma unroll
    for (int i = 0; i < T::NL; ++i) load_one(j, i);
  }
  if constexpr (T::kLate) {
    __builtin_amdgcn_s_waitcnt(waitcnt_imm(T::NL, 0));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  } else {
    stage_barrier();
  }
#pragma unroll
  for (int i = 0; i < T::TM; ++i) read_u(smU[0], fu0, 0, i);
#pragma unroll
  for (int i = 0; i < kVReads; ++i) read_v(smV[0], fv0, 0, i);
  int32_t s = 0;
  for (; s + NS <= ksteps; s += NS) {
#pragma unroll
    for (int j = 0; j < NS; ++j) step(j, s + j);
  }
#pragma unroll
  for (int j = 0; j < NS - 1; ++j)
    if (s + j < ksteps) step(j, s + j);

  if (part >= 0) {
    f32x4* to = reinterpret_cast<f32x4*>(p.part + (int64_t)part * (BM * BN));
#pragma unroll
    for (int mt = 0; mt < T::TM; ++mt)
#pragma unroll
      for (int nt = 0; nt < T::TN; ++nt) to[frag_index<T::TM, T::TN, 1>(wave, mt, nt, 0, lane)] = acc[mt][nt];
    return;
  }
  // Epilogue: through the stage buffers, so that whole lines are stored.
  __builtin_amdgcn_s_waitcnt(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  const StagedTile<BM, BN> t{smU[0], smV[0]};
  if (p.D) {
    if constexpr (kEarly) early.put(t, 0, tid);
    else ns_copy_in<BM, BN, T::THREADS>(p, t, mat, ti * BM, tj * BN, tid);
    staged_barrier();
  }
#pragma unroll
  for (int mt = 0; mt < T::TM; ++mt)
#pragma unroll
    for (int nt = 0; nt < T::TN; ++nt)
      {
        const int r = wm * T::WM + 16 * mt + (lane & 15), c = wn * T::WN + 16 * nt + 4 * (lane >> 4);
        ns_combine<SYM>(p, t.at(r, c), acc[mt][nt], ti * BM + r, tj * BN + c);
      }
  staged_barrier();
  ns_store<BM, BN, SYM>(p, t, mat, ti * BM, tj * BN, ti != tj, tid);
#endif
}

// The split tiles: ranges summed in order. A workgroup takes 32 rows of a tile
// (two rows of 16x16 tiles of one row of waves), or a whole one of 64.
template <int B, bool SYM>
__global__ void __launch_bounds__(512) ns_split_sum_kernel(NsParams p) {
  using T = NsTile<B, B, true, 2>;
  constexpr int ROWS = B == 64 ? 64 : 32, PARTS = B / ROWS;
  constexpr int R16 = ROWS / 16, FRAGS = R16 * B / 16;       // 16x16 tiles of a column, of a part
  __shared__ __attribute__((aligned(16))) char sm[ROWS * B * 2];
  const int32_t tile = blockIdx.x / PARTS, row0 = blockIdx.x % PARTS * ROWS;
  const int32_t id = p.whole + tile, mat = id / p.tiles;
  int32_t ti, tj;
  ns_tile<SYM>(p, id - mat * p.tiles, &ti, &tj);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const StagedTile<ROWS, B> t{sm, sm + ROWS * B};
  if (p.D) {
    ns_copy_in<ROWS, B, 512>(p, t, mat, ti * B + row0, tj * B, tid);
    __syncthreads();
  }
  const f32x4* from = reinterpret_cast<const f32x4*>(p.part + (int64_t)tile * p.splits * (B * B));
#pragma unroll
  for (int i = 0; i < FRAGS / 8; ++i) {
    const int f = wave * (FRAGS / 8) + i, row = f % R16 * 16, col = f / R16;
    const int w = (row0 + row) / T::WM * T::WGN + col / T::TN;               // the wave that computed it
    const int at = frag_index<T::TM, T::TN, 1>(w, (row0 + row) % T::WM / 16, col % T::TN, 0, lane);
    f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int r = 0; r < p.splits; ++r) v += from[(int64_t)r * (B * B / 4) + at];
    const int r = row + (lane & 15), c = 16 * col + 4 * (lane >> 4);
    ns_combine<SYM>(p, t.at(r, c), v, ti * B + row0 + r, tj * B + c);
  }
  __syncthreads();
  ns_store<ROWS, B, SYM>(p, t, mat, ti * B + row0, tj * B, ti != tj, tid);
}

// ---- the norm and the first X ----

struct NsInput {
  const void* G;
  int64_t ld, stride;       // elements
  int64_t rows, cols;
  int32_t f32;
  double* part;             // [matrices][chunks] sums of squares
  int32_t chunks;
  uint16_t* X;              // fp16 pp x qp
  int64_t x_stride;
  int32_t pp, qp, ld_x, tall;
  float eps;
};

// Eight elements of a row from column c, zeros past the last.
__device__ __forceinline__ void ns_load8(const NsInput& p, int64_t mat, int64_t r, int64_t c, float (&v)[8]) {
  const int64_t at = mat * p.stride + r * p.ld + c;
  const bool whole = c + 8 <= p.cols;
  if (p.f32) {
    const float* g = static_cast<const float*>(p.G) + at;
    if (whole && (reinterpret_cast<uintptr_t>(g) & 15) == 0) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(g), b = *reinterpret_cast<const f32x4*>(g + 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) { v[j] = a[j]; v[4 + j] = b[j]; }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = c + j < p.cols ? g[j] : 0.f;
    }
  } else {
    const uint16_t* g = static_cast<const uint16_t*>(p.G) + at;
    if (whole && (reinterpret_cast<uintptr_t>(g) & 15) == 0) {
      const uint4 a = *reinterpret_cast<const uint4*>(g);
      const f32x4 lo = bf16x4_to_f32(make_uint2(a.x, a.y)), hi = bf16x4_to_f32(make_uint2(a.z, a.w));
#pragma unroll
      for (int j = 0; j < 4; ++j) { v[j] = lo[j]; v[4 + j] = hi[j]; }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = c + j < p.cols ? __uint_as_float((uint32_t)g[j] << 16) : 0.f;
    }
  }
}

// Sum over the workgroup (256 threads), in every thread, in a fixed order.
__device__ __forceinline__ double block_sum(double v, double* sm) {
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) v += __shfl_xor(v, x);
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
  __syncthreads();
  return ((sm[0] + sm[1]) + sm[2]) + sm[3];
}

// Squares in fp64: neither a square nor the sum can over- or underflow.
__global__ void __launch_bounds__(256) ns_square_kernel(NsInput p) {
  __shared__ double sm[4];
  const int64_t mat = blockIdx.x / p.chunks, chunk = blockIdx.x - mat * p.chunks;
  const int64_t per_row = (p.cols + 7) / 8, units = per_row * p.rows;
  double sum = 0.0;
  for (int64_t u = chunk * 256 + threadIdx.x; u < units; u += (int64_t)p.chunks * 256) {
    const int64_t r = u / per_row;
    float v[8];
    ns_load8(p, mat, r, (u - r * per_row) * 8, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum = __builtin_fma((double)v[j], (double)v[j], sum);
  }
  sum = block_sum(sum, sm);
  if (threadIdx.x == 0) p.part[mat * p.chunks + chunk] = sum;
}

// X = fp16(kScale G / (|G| + eps)), 64 x 64 elements of X a workgroup, through
// LDS where X is G's transpose.
__global__ void __launch_bounds__(256) ns_first_kernel(NsInput p) {
  __shared__ double sm[4];
  __shared__ __attribute__((aligned(16))) uint16_t st[64][72];
  const int32_t tiles_c = p.qp / 64, tiles = p.pp / 64 * tiles_c;
  const int64_t mat = blockIdx.x / tiles;
  const int32_t t = blockIdx.x - mat * tiles, tr = t / tiles_c, tc = t - tr * tiles_c;
  double sum = 0.0;
  for (int i = threadIdx.x; i < p.chunks; i += 256) sum += p.part[mat * p.chunks + i];
  sum = block_sum(sum, sm);
  // The factor as m 2^e, m in [1/2, 1]: the inverse of a norm may be past fp32's
  // largest, or subnormal, where G times it is not. A zero G: zeros, with no eps too.
  int e;
  const float m = (float)frexp(sum == 0.0 ? 0.0 : kScale / (sqrt(sum) + (double)p.eps), &e);
  // the tile in G: rows g_r .., columns g_c ..
  const int64_t g_r = 64 * (int64_t)(p.tall ? tc : tr), g_c = 64 * (int64_t)(p.tall ? tr : tc);
  uint16_t* X = p.X + mat * p.x_stride + 64 * (int64_t)tr * p.ld_x + 64 * tc;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int at = i * 256 + threadIdx.x, r = at >> 3, c = (at & 7) * 8;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (g_r + r < p.rows && g_c + c < p.cols) ns_load8(p, mat, g_r + r, g_c + c, v);
    f16x8 o;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = (_Float16)(ldexpf(v[j], e) * m);
    if (!p.tall) {
      *reinterpret_cast<f16x8*>(X + (int64_t)r * p.ld_x + c) = o;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const _Float16 e = o[j];
        st[c + j][r] = __builtin_bit_cast(uint16_t, e);
      }
    }
  }
  if (!p.tall) return;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int at = i * 256 + threadIdx.x, r = at >> 3, c = (at & 7) * 8;
    *reinterpret_cast<uint4*>(X + (int64_t)r * p.ld_x + c) = *reinterpret_cast<const uint4*>(&st[r][c]);
  }
}

// No steps: the scaled G itself, O = X / kScale.
__global__ void __launch_bounds__(256) ns_copy_kernel(const uint16_t* X, int64_t x_stride, int32_t ldx, uint16_t* O,
                                                      int64_t o_stride, int64_t o_ld, int64_t rows, int64_t cols,
                                                      int32_t tall) {
  const int64_t n = rows * cols, blocks = (n + 255) / 256;
  const int64_t mat = blockIdx.x / blocks, i = (blockIdx.x - mat * blocks) * 256 + threadIdx.x;
  if (i >= n) return;
  const int64_t r = i / cols, c = i - r * cols;
  const float v = (float)__builtin_bit_cast(_Float16, X[mat * x_stride + (tall ? c * ldx + r : r * ldx + c)]);
  O[mat * o_stride + r * o_ld + c] = __builtin_bit_cast(uint16_t, (__bf16)(v / kScale));
}

// One product of the batch.
template <bool SYM>
hipError_t ns_launch(NsParams p, int64_t batch, const OrthoSplit& f, hipStream_t stream) {
  const int b = f.tile, bn = b == 64 && !SYM ? 128 : b;
  p.tiles_m = (p.M + b - 1) / b;
  p.tiles_n = (p.N + bn - 1) / bn;
  p.tiles = SYM ? p.tiles_m * (p.tiles_m + 1) / 2 : p.tiles_m * p.tiles_n;
  p.total = (int32_t)(p.tiles * batch);
  p.group = p.tiles_m < 8 ? p.tiles_m : 8;
  p.whole = f.whole;
  p.splits = f.splits;
  p.ksplit = f.ksplit;
  p.whole_xcd = (f.whole + 7) / 8;
  const int32_t rest = p.total - p.whole;
  p.split_xcd = (rest * f.splits + 7) / 8;
  const dim3 grid((unsigned)(8 * (p.whole_xcd + p.split_xcd))), block(512);
  if (b == 64) hipLaunchKernelGGL((ns_product_kernel<64, SYM ? 64 : 128, SYM, 4>), grid, block, 0, stream, p);
  else if (b == 128 && f.paired) hipLaunchKernelGGL((ns_product_kernel<128, 128, SYM, 2>), grid, block, 0, stream, p);
  else if (b == 128) hipLaunchKernelGGL((ns_product_kernel<128, 128, SYM, 4>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((ns_product_kernel<256, 256, SYM, 2>), grid, block, 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || rest == 0) return e;
  if (b == 64) hipLaunchKernelGGL((ns_split_sum_kernel<64, true>), dim3((unsigned)rest), block, 0, stream, p);
  else if (b == 128) hipLaunchKernelGGL((ns_split_sum_kernel<128, SYM>), dim3((unsigned)(rest * 4)), block, 0, stream, p);
  else hipLaunchKernelGGL((ns_split_sum_kernel<256, SYM>), dim3((unsigned)(rest * 8)), block, 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_orthogonalize(const OrthoShape& s, const OrthoCall& c, void* ws, hipStream_t stream) {
  const OrthoForm f = ortho_form(s);
  char* base = static_cast<char*>(ws);
  const auto at = [&](int64_t offset) { return reinterpret_cast<uint16_t*>(base + offset); };
  uint16_t *S = at(f.s_at), *B = at(f.b_at);
  uint16_t* x[2] = {at(f.x_at[0]), at(f.x_at[1])};
  const bool tall = s.rows > s.cols;

  NsInput in;
  in.G = c.G;
  in.ld = c.ld;
  in.stride = c.stride;
  in.rows = s.rows;
  in.cols = s.cols;
  in.f32 = c.f32 ? 1 : 0;
  in.part = reinterpret_cast<double*>(base);
  in.chunks = f.chunks;
  in.X = x[0];
  in.x_stride = f.x_elems;
  in.pp = f.pp;
  in.qp = f.qp;
  in.ld_x = f.ld_q;
  in.tall = tall ? 1 : 0;
  in.eps = c.eps;
  hipLaunchKernelGGL(ns_square_kernel, dim3((unsigned)(f.chunks * s.batch)), dim3(256), 0, stream, in);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(ns_first_kernel, dim3((unsigned)((int64_t)f.pp / 64 * (f.qp / 64) * s.batch)), dim3(256), 0, stream, in);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (c.steps == 0) {
    const int64_t blocks = (s.rows * s.cols + 255) / 256 * s.batch;
    hipLaunchKernelGGL(ns_copy_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, x[0], f.x_elems, f.ld_q,
                       static_cast<uint16_t*>(c.O), c.o_stride, c.o_ld, s.rows, s.cols, in.tall);
    return hipGetLastError();
  }
  // S comes near I: B is held less its value there, whose rounding on the
  // diagonal was the largest of the errors (100x100: 1.7e-3 of the result, now
  // 1.4e-3). Larger values gain nothing and might overflow.
  const float at_one = -(c.coeffs[1] + c.coeffs[2]);
  const float shift = at_one > -4.f && at_one < 4.f ? at_one : 0.f;
  for (int step = 0; step < c.steps; ++step) {
    const uint16_t* X = x[step & 1];
    const bool last = step + 1 == c.steps;
    NsParams p{};
    p.part = reinterpret_cast<float*>(base + f.part_at);
    p.o_ld = c.o_ld;
    p.o_stride = c.o_stride;
    p.o_rows = (int32_t)s.rows;
    p.o_cols = (int32_t)s.cols;
    // S = X X^T
    p.U = p.V = X;
    p.u_stride = p.v_stride = f.x_elems;
    p.ldu = p.ldv = f.ld_q;
    p.out = S;
    p.out_stride = f.s_elems;
    p.ld_out = f.ld_p;
    p.M = p.N = f.pp;
    p.K = f.qp;
    p.alpha = 1.f / kScale;
    if ((e = ns_launch<true>(p, s.batch, f.gram, stream)) != hipSuccess) return e;
    // B = b S + c S S + s I (S is its own transpose)
    p.U = p.V = p.D = S;
    p.u_stride = p.v_stride = f.s_elems;
    p.ldu = p.ldv = f.ld_p;
    p.out = B;
    p.K = f.pp;
    p.alpha = c.coeffs[2] / kScale;
    p.beta = c.coeffs[1];
    p.diag = kScale * shift;
    if ((e = ns_launch<true>(p, s.batch, f.square, stream)) != hipSuccess) return e;
    // X <- (a - s) X + B X
    p.diag = 0.f;
    p.U = B;
    p.V = p.D = X;
    p.v_stride = f.x_elems;
    p.ldv = f.ld_q;
    p.out = x[(step + 1) & 1];
    p.out_stride = f.x_elems;
    p.ld_out = f.ld_q;
    p.N = f.qp;
    p.o_trans = in.tall;
    p.O = last ? static_cast<uint16_t*>(c.O) : nullptr;
    p.alpha = last ? 1.f / (kScale * kScale) : 1.f / kScale;
    p.beta = (c.coeffs[0] - shift) / (last ? kScale : 1.f);
    e = ns_launch<false>(p, s.batch, f.update, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace ccl
