// Tiles of a bf16 product D = U V' with fp32 sums, for operands that are
// stored either way round: each side's rows may have K contiguous ("KC": X and
// output-major weights of Y = X W^T) or be the columns of a matrix whose rows
// are K ("RC": W in dX = dY W; both sides in dW = dY^T X). The experts'
// products and the vocabulary loss are built on it.
//
// A workgroup of 8 waves computes BM x BN. A stage is 64 K: KC rows lie in LDS
// as 128-byte rows (chunk c of row r at c ^ swz_a64(r)) and are read with
// ds_read_b128; RC ones as 64 rows of BM or BN with the transposing reads. The
// K loop is the one of the GEMM's 64-K tiles: the MFMAs of a stage's two halves
// around one barrier, the next half's fragments read behind them.
//
// Bounds: rows past a KC side's extent and K rows past its end come from
// outside the descriptor and read as zeros (its length is set stage by stage,
// so the operands may be of any size), chunks of a KC row past K are sent past
// it too. Columns past an RC side's extent hold other values of the matrix, but
// reach only rows or columns of D that are not stored.
#pragma once

#include "gemm_tiles.hpp"

namespace ccl {

namespace {

// One side of a tile: the address of its first row (KC) or column (RC) at K =
// 0, elements between memory rows, valid rows (KC) or columns (RC) of the
// tile, and the K that are there. Uniform over the workgroup.
struct Side {
  const uint16_t* base;
  int64_t ld;
  int32_t extent;
  int32_t k;
};

template <int BM_, int BN_, bool UK_, bool VK_, int NS_, int WGN_ = 4>
struct ProductTile {
  static constexpr int BM = BM_, BN = BN_, NS = NS_, WGN = WGN_;
  static constexpr bool UK = UK_, VK = VK_;
  static constexpr int NW = 8, THREADS = 512, WGM = NW / WGN;
  static constexpr int WM = BM / WGM, WN = BN / WGN, TM = WM / 16, TN = WN / 16;
  static constexpr int U_BYTES = BM * 128, V_BYTES = BN * 128;
  static constexpr int NU = U_BYTES / (1024 * NW), NV = V_BYTES / (1024 * NW), NL = NU + NV;
  static constexpr int LDS = NS * (U_BYTES + V_BYTES);
  // With two stage buffers a step's loads go out behind its barrier, into the
  // buffer it has just read; otherwise NS - 1 stages ahead of it.
  static constexpr bool kLate = NS == 2;
  static constexpr int AHEAD = kLate ? 2 : NS - 1;
  static_assert(NU >= 1 && NV >= 1 && NU <= 4 && NV <= 4, "a run of loads shares one M0");
  static_assert(TM >= 1 && TN >= 1 && NS >= 2 && LDS <= 160 * 1024, "tile");
};

// The loads of one side: per-lane offsets and the stage that comes next.
template <int B, bool KC, int N>
struct SideLoads {
  // Load i of a run lands 1024 i bytes on through its instruction offset, which
  // moves its memory address too: the per-lane offsets are less by as much,
  // and the descriptor starts kShift early to keep them positive.
  static constexpr uint32_t kShift = 1024 * (N - 1);
  static constexpr int CPR = B / 8, RPI = 64 / CPR;     // RC: chunks of a row, rows of a load
  uint32_t voff[N];
  uint64_t at;
  int64_t step;            // bytes from one stage to the next
  int64_t ld2;             // bytes between rows
  int32_t extent, left;    // left: K from the next stage on
  int wave, lane;

  __device__ __forceinline__ static int row(int wave, int lane, int i) {
    return KC ? 8 * (wave * N + i) + (lane >> 3) : RPI * (wave * N + i) + lane / CPR;
  }
  __device__ __forceinline__ static int chunk(int wave, int lane, int i) {
    const int r = row(wave, lane, i);
    return KC ? (lane & 7) ^ swz_a64(r) : (lane % CPR) ^ swz_bn<B>(r);
  }
  // map: the memory row of a KC tile row.
  template <typename Map>
  __device__ __forceinline__ void init(const Side& s, int32_t k0, int w, int l, Map&& map) {
    wave = w;
    lane = l;
    ld2 = s.ld * 2;
    extent = s.extent;
    left = s.k - k0;
    step = KC ? 128 : 64 * ld2;
    at = reinterpret_cast<uint64_t>(s.base) + (KC ? (int64_t)k0 * 2 : (int64_t)k0 * ld2) - kShift;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = row(w, l, i);
      voff[i] = (uint32_t)((KC ? map(r) : r) * ld2) + chunk(w, l, i) * 16u + kShift - 1024u * i;
    }
  }
  // The descriptor of the next stage (of no memory past the last).
  __device__ __forceinline__ i32x4 next() {
    int32_t bytes = 0;
    if (left > 0) {
      const int32_t k = min(left, 64);
      bytes = KC ? (int32_t)((extent - 1) * ld2) + 2 * k : (int32_t)((k - 1) * ld2) + 2 * extent;
      bytes += kShift;
      if (KC && left < 64) {
        // the last stage, of fewer K: the other chunks of a row lie past everything
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (8 * chunk(wave, lane, i) >= left) voff[i] = 0x80000000u;
      }
    }
    i32x4 d;
    d[0] = (int)(uint32_t)at;
    d[1] = (int)((at >> 32) & 0xffffu);
    d[2] = bytes;
    d[3] = 0x00020000;
    at += step;
    left -= 64;
    return d;
  }
  __device__ __forceinline__ void load(const i32x4& d, char* lds, int i) const {
    lds_dma16_run<false>(d, voff[i], 0u, lds + (wave * N + i) * 1024, i);
  }
};

// The fragments of one side in a stage's half kk: 16 x 32 tiles, lane l with
// row l % 16 and K 8 (l / 16) .. + 7.
template <int B, bool KC, int T, int W>
struct SideFrags {
  static constexpr int READS = KC ? T : 2 * T;
  bf16x8 k[KC ? T : 1];
  i16x4 r[KC ? 1 : T][2];
  // Byte offset of the wave's first tile; w0: the wave's first row or column.
  __device__ __forceinline__ static int32_t first(int w0, int lane) {
    if constexpr (KC) {
      const int row = w0 + (lane & 15);
      return row * 128 + (((lane >> 4) ^ swz_a64(row)) * 16);
    } else {
      const int g = lane >> 4, s = lane & 15, krow = 8 * g + (s >> 2), col = w0 + 4 * (s & 3);
      return krow * (B * 2) + (((col >> 3) ^ swz_bn<B>(krow)) * 16) + ((col >> 2) & 1) * 8;
    }
  }
  // Read i of READS. KC: half kk of a row is the chunk with bit 2 flipped. RC:
  // a tile's columns start 32 bytes after the last one's, below the wave's
  // width, so its chunk is the first tile's XOR that; rows 4 on have the same
  // swizzle.
  __device__ __forceinline__ void read(const char* lds, int32_t first, int kk, int i) {
    if constexpr (KC) {
      k[i] = *(const lds_bf16x8*)(lds + (first ^ (kk * 64)) + i * 16 * 128);
    } else {
      static_assert((W & (W - 1)) == 0, "the wave's columns start at a multiple of their number");
      const int t = i >> 1, h = i & 1;
      r[t][h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_i16x4*)(lds + (first ^ (t * 32)) + h * 4 * B * 2 + kk * 32 * B * 2));
    }
  }
  __device__ __forceinline__ bf16x8 get(int t) const {
    if constexpr (KC) return k[t];
    else return __builtin_bit_cast(bf16x8, __builtin_shufflevector(r[t][0], r[t][1], 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

#if defined(__HIP_DEVICE_COMPILE__)
// acc = U V' over K [k0, ...) of ksteps stages of 64 (at least one). sm: T::LDS
// bytes, 1024-byte aligned, free when this returns. vmap: the memory row of a
// KC V tile row.
template <typename T, typename VMap>
__device__ __forceinline__ void product(const Side& u, const Side& v, int32_t k0, int32_t ksteps,
                                        f32x4 (&acc)[T::TM][T::TN], char* sm, int tid, VMap&& vmap) {
  constexpr int NS = T::NS;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / T::WGN, wn = wave % T::WGN;
  char* const smU = sm;
  char* const smV = sm + NS * T::U_BYTES;
  SideLoads<T::BM, T::UK, T::NU> lu;
  SideLoads<T::BN, T::VK, T::NV> lv;
  lu.init(u, k0, wave, lane, [](int r) { return r; });
  lv.init(v, k0, wave, lane, vmap);
  using FU = SideFrags<T::BM, T::UK, T::TM, T::WM>;
  using FV = SideFrags<T::BN, T::VK, T::TN, T::WN>;
  FU fu0, fu1;
  FV fv0, fv1;
  const int32_t u_rd = FU::first(wm * T::WM, lane), v_rd = FV::first(wn * T::WN, lane);
#pragma unroll
  for (int i = 0; i < T::TM; ++i)
#pragma unroll
    for (int j = 0; j < T::TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto mfma_one = [&](const FU& fu, const FV& fv, int i) __attribute__((always_inline)) {
    const int mt = i / T::TN, nt = i % T::TN;
    acc[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fv.get(nt), fu.get(mt), acc[mt][nt], 0, 0, 0);
  };
  auto load_one = [&](const i32x4& du, const i32x4& dv, int at, int i) __attribute__((always_inline)) {
    if (i < T::NU) lu.load(du, smU + at * T::U_BYTES, i);
    else lv.load(dv, smV + at * T::V_BYTES, i - T::NU);
  };
  constexpr int kReads = FU::READS + FV::READS;
  auto read_one = [&](FU& fu, FV& fv, int at, int kk, int i) __attribute__((always_inline)) {
    if (i < FU::READS) fu.read(smU + at * T::U_BYTES, u_rd, kk, i);
    else fv.read(smV + at * T::V_BYTES, v_rd, kk, i - FU::READS);
  };
  auto stage_barrier = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(waitcnt_imm((NS - 2) * T::NL, 0));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // A step on stage buffer ph; on entry fu0 / fv0 hold its first half.
  auto step = [&](int ph) __attribute__((always_inline)) {
    constexpr int kMfma = T::TM * T::TN;
    constexpr int kOps1 = kReads + (T::kLate ? 0 : T::NL), kAll1 = kMfma > kOps1 ? kMfma : kOps1;
    const i32x4 du = lu.next(), dv = lv.next();
    const int to = (ph + T::AHEAD) % NS, nx = (ph + 1) % NS;
#pragma unroll
    for (int i = 0; i < kAll1; ++i) {
      if (i < kMfma) mfma_one(fu0, fv0, i);
      if (i < kReads) read_one(fu1, fv1, ph, 1, i);
      else if (i < kOps1) load_one(du, dv, to, i - kReads);
      __builtin_amdgcn_sched_barrier(0);
    }
    stage_barrier();
    constexpr int kOps2 = T::kLate && T::NL > kReads ? T::NL : kReads, kAll2 = kMfma > kOps2 ? kMfma : kOps2;
#pragma unroll
    for (int i = 0; i < kAll2; ++i) {
      if (i < kMfma) mfma_one(fu1, fv1, i);
      if (i < kReads) read_one(fu0, fv0, nx, 0, i);
      if (T::kLate && i < T::NL) load_one(du, dv, to, i);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

#pragma unroll
  for (int j = 0; j < T::AHEAD; ++j) {
    const i32x4 du = lu.next(), dv = lv.next();
#pragma unroll
    for (int i = 0; i < T::NL; ++i) load_one(du, dv, j, i);
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
  for (int i = 0; i < kReads; ++i) read_one(fu0, fv0, 0, 0, i);
  int32_t s = 0;
  for (; s + NS <= ksteps; s += NS) {
#pragma unroll
    for (int j = 0; j < NS; ++j) step(j);
  }
#pragma unroll
  for (int j = 0; j < NS - 1; ++j)
    if (s + j < ksteps) step(j);
  // loads past the last stage write zeros to LDS: they land before it is reused
  __builtin_amdgcn_s_waitcnt(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
#endif

// Tiles are dealt to the XCDs (workgroup mod 8) in runs of chunk, so that what
// runs on one XCD together shares operands in its L2 and uneven experts spread.
__device__ __forceinline__ int64_t dealt_tile(int32_t chunk) {
  const uint32_t xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
  const uint32_t run = slot / (uint32_t)chunk;
  return ((int64_t)run * 8 + xcd) * chunk + (slot - run * chunk);
}

// The staged tile's rows < rows and chunks with col(chunk) >= 0 to m.
template <int ROWS, int COLS, int THREADS, typename Col>
__device__ __forceinline__ void tile_out(const StagedTile<ROWS, COLS>& t, uint16_t* m, int64_t ld, int32_t rows, int tid,
                                         Col&& col) {
  constexpr int CPR = COLS / 8;
#pragma unroll 4
  for (int i = 0; i < ROWS * CPR / THREADS; ++i) {
    const int at = i * THREADS + tid, r = at / CPR, c = at % CPR;
    const uint4 v = *reinterpret_cast<const uint4*>(t.chunk(r, c));
    const int32_t to = col(c);
    if (r < rows && to >= 0) *reinterpret_cast<uint4*>(m + r * ld + to) = v;
  }
}

template <int ROWS, int COLS, int THREADS, typename Col>
__device__ __forceinline__ void tile_in(const StagedTile<ROWS, COLS>& t, const uint16_t* m, int64_t ld, int32_t rows, int tid,
                                        Col&& col) {
  constexpr int CPR = COLS / 8, N = ROWS * CPR / THREADS, B = N < 8 ? N : 8;
  for (int i = 0; i < N; i += B) {
    uint4 v[B];
#pragma unroll
    for (int j = 0; j < B; ++j) {
      const int at = (i + j) * THREADS + tid, r = at / CPR;
      const int32_t from = col(at % CPR);
      v[j] = make_uint4(0, 0, 0, 0);
      if (r < rows && from >= 0) v[j] = *reinterpret_cast<const uint4*>(m + r * ld + from);
    }
#pragma unroll
    for (int j = 0; j < B; ++j) {
      const int at = (i + j) * THREADS + tid;
      *reinterpret_cast<uint4*>(t.chunk(at / CPR, at % CPR)) = v[j];
    }
  }
}

// A tile's values in a lane's order: f(mt, nt, row, column of its four).
template <typename T, typename F>
__device__ __forceinline__ void each4(int tid, F&& f) {
  const int lane = tid & 63, wave = tid >> 6, wm = wave / T::WGN, wn = wave % T::WGN;
#pragma unroll
  for (int mt = 0; mt < T::TM; ++mt)
#pragma unroll
    for (int nt = 0; nt < T::TN; ++nt) f(mt, nt, wm * T::WM + 16 * mt + (lane & 15), wn * T::WN + 16 * nt + 4 * (lane >> 4));
}

template <int BM, int BN>
__device__ __forceinline__ StagedTile<BM, BN> staged(char* sm) {
  return StagedTile<BM, BN>{sm, sm + BM / 2 * BN * 2};
}

}  // namespace

}  // namespace ccl
