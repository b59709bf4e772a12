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
// so the operands may be of any size); chunks of a KC row past K, in a last
// part of a stage, are sent past it too. Columns past an RC side's extent hold other values of the matrix, but
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
  int wave;

  __device__ __forceinline__ static int row(int wave, int lane, int i) {
    return KC ? 8 * (wave * N + i) + (lane >> 3) : RPI * (wave * N + i) + lane / CPR;
  }
  __device__ __forceinline__ static int chunk(int wave, int lane, int i) {
    const int r = row(wave, lane, i);
    return KC ? (lane & 7) ^ swz_a64(r) : (lane % CPR) ^ swz_bn<B>(r);
  }
  // map: the memory row of a KC tile row. chunks: of a KC stage row that exist,
  // the others are sent past everything.
  template <typename Map>
  __device__ __forceinline__ void init(const Side& s, int32_t k0, int w, int l, Map&& map, int chunks = 8) {
    wave = w;
    ld2 = s.ld * 2;
    extent = s.extent;
    left = s.k - k0;
    step = KC ? 128 : 64 * ld2;
    at = reinterpret_cast<uint64_t>(s.base) + (KC ? (int64_t)k0 * 2 : (int64_t)k0 * ld2) - kShift;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = row(w, l, i), c = chunk(w, l, i);
      voff[i] = (uint32_t)((KC ? map(r) : r) * ld2) + c * 16u + kShift - 1024u * i;
      if (KC && c >= chunks) voff[i] = 0x80000000u;
    }
  }
  // The descriptor of the next stage (of no memory past the last).
  __device__ __forceinline__ i32x4 next() {
    int32_t bytes = 0;
    if (left > 0) {
      const int32_t k = min(left, 64);
      bytes = (KC ? (int32_t)((extent - 1) * ld2) + 2 * k : (int32_t)((k - 1) * ld2) + 2 * extent) + (int32_t)kShift;
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

// A fragment of one side in a stage's half kk: 16 x 32 of a wave's T tiles, lane l
// with row l % 16 and K 8 (l / 16) .. + 7.
template <int B, bool KC, int T>
struct SideFrag {
  static constexpr int READS = KC ? 1 : 2;
  bf16x8 k;
  i16x4 r[2];
  // Addresses that its reads start from, the rest being constants: KC: of the
  // halves (half 1 of a row is the chunk with bit 2 flipped); RC: of the tiles (a
  // tile's columns start 32 bytes after the last one's, below the wave's width, so
  // its chunk is the first tile's XOR that; rows 4 on have the same swizzle). Kept
  // from the compiler, which would form and spill one for every read.
  static constexpr int NA = KC ? 2 : T;
  static_assert(KC || (T & (T - 1)) == 0, "the wave's columns start at a multiple of their number");
  // w0: the wave's first row or column.
  __device__ __forceinline__ static void addresses(const char* lds, int w0, int lane, uint32_t (&at)[NA]) {
    uint32_t first;
    if constexpr (KC) {
      const int row = w0 + (lane & 15);
      first = row * 128 + (((lane >> 4) ^ swz_a64(row)) * 16);
    } else {
      const int g = lane >> 4, s = lane & 15, krow = 8 * g + (s >> 2), col = w0 + 4 * (s & 3);
      first = krow * (B * 2) + (((col >> 3) ^ swz_bn<B>(krow)) * 16) + ((col >> 2) & 1) * 8;
    }
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      at[i] = (uint32_t)(uintptr_t)(const lds_char*)lds + (first ^ (KC ? i * 64 : i * 32));
      asm volatile("" : "+v"(at[i]));
    }
  }
  // Read h of tile t, in the stage buffer `stage` bytes on.
  __device__ __forceinline__ void read(const uint32_t (&at)[NA], int stage, int kk, int t, int h) {
    if constexpr (KC) {
      k = *(const lds_bf16x8*)(uintptr_t)(at[kk] + stage + t * 16 * 128);
    } else {
      r[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_i16x4*)(uintptr_t)(at[t] + stage + h * 4 * B * 2 + kk * 32 * B * 2));
    }
  }
  __device__ __forceinline__ bf16x8 get() const {
    if constexpr (KC) return k;
    else return __builtin_bit_cast(bf16x8, __builtin_shufflevector(r[0], r[1], 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

#if defined(__HIP_DEVICE_COMPILE__)
// acc = U V' over K [k0, ...) of ksteps stages of 64 (at least one), the last of
// which may be part of one. sm: T::LDS bytes, 1024-byte aligned, free when this
// returns. vmap: the memory row of a KC V tile row.
//
// A half's MFMAs go tile row by tile row of U: as soon as a row's are issued, its
// fragment's registers take the next half's. The last two rows and V have two
// sets, read first, so that every read of a stage is a good part of a half old at
// the barrier (whole second sets of U too would not fit beside a 256x256 tile's
// accumulators).
template <typename T, typename VMap>
__device__ __forceinline__ void product(Side u, Side v, int32_t k0, int32_t ksteps, f32x4 (&acc)[T::TM][T::TN], char* sm,
                                        int tid, VMap&& vmap) {
  constexpr int NS = T::NS, TM = T::TM, TN = T::TN;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / T::WGN, wn = wave % T::WGN;
  char* const smV = sm;
  char* const smU = sm + NS * T::V_BYTES;
  using LU = SideLoads<T::BM, T::UK, T::NU>;
  using LV = SideLoads<T::BN, T::VK, T::NV>;
  using FU = SideFrag<T::BM, T::UK, TM>;
  using FV = SideFrag<T::BN, T::VK, TN>;
  constexpr int SP = TM < 2 ? TM : 2, KEPT = TM - SP;    // rows of U with two sets, and with one
  FU fu[KEPT ? KEPT : 1], fs[2][SP];
  FV fv[2][TN];
  uint32_t ua[FU::NA], va[FV::NA];
  FU::addresses(smU, wm * T::WM, lane, ua);
  FV::addresses(smV, wn * T::WN, lane, va);
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Part of a stage where chunks of K-contiguous rows end: apart, behind the loop.
  const int32_t end = T::UK ? u.k : v.k;
  const int32_t rest = (T::UK || T::VK) && k0 + ksteps * 64 > end ? end & 63 : 0;
  if (rest) --ksteps;
  const Side u_all = u, v_all = v;
  u.k = min(u.k, k0 + ksteps * 64);
  v.k = min(v.k, k0 + ksteps * 64);

  auto mfma_one = [&](int set, int i) __attribute__((always_inline)) {
    const int mt = i / TN, nt = i % TN;
    const bf16x8 a = mt < KEPT ? fu[mt < KEPT ? mt : 0].get() : fs[set][mt < KEPT ? 0 : mt - KEPT].get();
    acc[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fv[set][nt].get(), a, acc[mt][nt], 0, 0, 0);
  };
  // Reads into the second sets: V's tiles and U's last rows, in this order.
  constexpr int kV = TN * FV::READS, kFirst = kV + SP * FU::READS;
  auto read_first = [&](int set, int ph, int kk, int i) __attribute__((always_inline)) {
    if (i < kV) fv[set][i / FV::READS].read(va, ph * T::V_BYTES, kk, i / FV::READS, i % FV::READS);
    else fs[set][(i - kV) / FU::READS].read(ua, ph * T::U_BYTES, kk, KEPT + (i - kV) / FU::READS, (i - kV) % FU::READS);
  };
  // One half on set `set`; behind its MFMAs the reads of the next one (half kk of
  // stage buffer ph) and `loads` further operations.
  auto half = [&](int set, int ph, int kk, int loads, auto&& load) __attribute__((always_inline)) {
    constexpr int kMfma = TM * TN;
    const int all = kFirst + loads > kMfma ? kFirst + loads : kMfma;
#pragma unroll
    for (int i = 0; i < all; ++i) {
      if (i < kMfma) mfma_one(set, i);
      if (i < kFirst) read_first(set ^ 1, ph, kk, i);
      else if (i < kFirst + loads) load(i - kFirst);
      if (i < kMfma && (i + 1) % TN == 0 && i / TN < KEPT) {
#pragma unroll
        for (int h = 0; h < FU::READS; ++h) fu[i / TN].read(ua, ph * T::U_BYTES, kk, i / TN, h);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto read_all = [&](int kk) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kFirst; ++i) read_first(0, 0, kk, i);
#pragma unroll
    for (int i = 0; i < KEPT; ++i)
#pragma unroll
      for (int h = 0; h < FU::READS; ++h) fu[i].read(ua, 0, kk, i, h);
  };
  auto barrier = [&](auto vm) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(waitcnt_imm(decltype(vm)::value, 0));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  if (ksteps > 0) {
    LU lu;
    LV lv;
    lu.init(u, k0, wave, lane, [](int r) { return r; });
    lv.init(v, k0, wave, lane, vmap);
    auto load_one = [&](const i32x4& du, const i32x4& dv, int at, int i) __attribute__((always_inline)) {
      if (i < T::NU) lu.load(du, smU + at * T::U_BYTES, i);
      else lv.load(dv, smV + at * T::V_BYTES, i - T::NU);
    };
    // A step on stage buffer ph; on entry set 0 holds its first half.
    auto step = [&](int ph) __attribute__((always_inline)) {
      const i32x4 du = lu.next(), dv = lv.next();
      const int to = (ph + T::AHEAD) % NS, nx = (ph + 1) % NS;
      auto load = [&](int i) __attribute__((always_inline)) { load_one(du, dv, to, i); };
      half(0, ph, 1, T::kLate ? 0 : T::NL, load);
      barrier(std::integral_constant<int, (NS - 2) * T::NL>{});
      half(1, nx, 0, T::kLate ? T::NL : 0, load);
    };
#pragma unroll
    for (int j = 0; j < T::AHEAD; ++j) {
      const i32x4 du = lu.next(), dv = lv.next();
#pragma unroll
      for (int i = 0; i < T::NL; ++i) load_one(du, dv, j, i);
    }
    barrier(std::integral_constant<int, T::kLate ? T::NL : (NS - 2) * T::NL>{});
    read_all(0);
    // One loop, left behind any step: with a second copy of the steps for what a
    // multiple of NS leaves over, the 256x256 tiles' accumulators were spilled.
    bool more = true;
    for (int32_t s = 0; more;) {
#pragma unroll
      for (int j = 0; j < NS; ++j)
        if (more) {
          step(j);
          more = ++s < ksteps;
        }
    }
    // loads past the last stage write zeros to LDS: they land before it is reused
    barrier(std::integral_constant<int, 0>{});
  }
  if (rest) {
    const int32_t k = k0 + ksteps * 64;
    LU lu;
    LV lv;
    lu.init(u_all, k, wave, lane, [](int r) { return r; }, rest / 8);
    lv.init(v_all, k, wave, lane, vmap, rest / 8);
    const i32x4 du = lu.next(), dv = lv.next();
#pragma unroll
    for (int i = 0; i < T::NU; ++i) lu.load(du, smU, i);
#pragma unroll
    for (int i = 0; i < T::NV; ++i) lv.load(dv, smV, i);
    barrier(std::integral_constant<int, 0>{});
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      read_all(kk);
#pragma unroll
      for (int i = 0; i < TM * TN; ++i) mfma_one(0, i);
    }
    barrier(std::integral_constant<int, 0>{});
  }
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
