// Tiles of a bf16 product D = U V' with fp32 sums, for operands that are
// stored either way round: each side's rows may have K contiguous ("KC": X and
// output-major weights of Y = X W^T) or be the columns of a matrix whose rows
// are K ("RC": W in dX = dY W; both sides in dW = dY^T X). The experts'
// products and the vocabulary loss are built on it.
//
// A workgroup computes BM x BN. A stage is 64 K: KC rows lie in LDS
// as 128-byte rows (chunk c of row r at c ^ swz_a64(r)) and are read with
// ds_read_b128; RC ones as 64 rows of BM or BN with the transposing reads. The
// MFMAs of a stage's two halves go around one barrier, the next half's fragments
// are read behind them.
//
// Workgroups stay and take tile after tile: the loads run through from one tile
// to the next, so that the next tile's first stages are on their way or there
// while a tile is finished and stored. (Products here are short: 4 stages of 64
// rows of an expert in dW, 12 to 32 of a hidden size; a workgroup that started
// with its tile waited 2 to 3 us for its first stage.)
//
// Bounds: rows past a KC side's extent and K rows past its end come from
// outside the descriptor and read as zeros (its length is set stage by stage,
// so the operands may be of any size); chunks of a KC row past K are sent past
// it too. Columns past an RC side's extent hold other values of the matrix, but
// reach only rows or columns of D that are not stored.
#pragma once

#include "gemm_tiles.hpp"

namespace ccl {

namespace {

// One side of a tile: the address of its first row (KC) or column (RC) at its
// first K, valid rows (KC) or columns (RC), and the K that are there. Uniform
// over the workgroup.
struct Side {
  const uint16_t* base;
  int32_t extent;
  int32_t k;
};

// BM x BN by NW waves, WGN of them along N; NS stages. SKIP: KC rows of U in 16-row tiles that
// lie past its extent are not multiplied. WHOLE: K of KC sides is a multiple of 64.
template <int BM_, int BN_, bool UK_, bool VK_, int NS_, int NW_, int WGN_, bool SKIP_ = false, bool WHOLE_ = false>
struct ProductTile {
  static constexpr int BM = BM_, BN = BN_, NS = NS_, WGN = WGN_;
  static constexpr bool UK = UK_, VK = VK_, SKIP = SKIP_, WHOLE = WHOLE_;
  static constexpr int NW = NW_, THREADS = 64 * NW, WGM = NW / WGN;
  static constexpr int WM = BM / WGM, WN = BN / WGN, TM = WM / 16, TN = WN / 16;
  static constexpr int U_BYTES = BM * 128, V_BYTES = BN * 128;
  static constexpr int NU = U_BYTES / (1024 * NW), NV = V_BYTES / (1024 * NW), NL = NU + NV;
  static constexpr int LDS = NS * (U_BYTES + V_BYTES);
  static constexpr int U_AT = 0, V_AT = NS * U_BYTES;
  // A stage's loads go into the buffer that the step has just read, behind its
  // barrier: NS stages ahead.
  static constexpr int AHEAD = NS;
  static_assert(NU >= 1 && NV >= 1 && NU <= 8 && NV <= 4, "loads");
  static_assert((UK || (BM & (BM - 1)) == 0) && (VK || (BN & (BN - 1)) == 0) && NS >= 2, "powers of two");
  static_assert(TM >= 1 && TN >= 1 && LDS <= 160 * 1024, "tile");
  static_assert(UK || !SKIP, "rows are skipped on a KC side");
  // Tile row mt of a wave, in rows of the tile. KC: a wave's rows are spread, so
  // that a tile with few valid rows keeps all waves at work.
  static constexpr int ROWS = UK ? 16 * WGM : 16;        // between a wave's tile rows
  __device__ static __forceinline__ int row(int wm, int mt) { return UK ? 16 * (WGM * mt + wm) : WM * wm + 16 * mt; }
};
// Waves a SIMD with the workgroups of a CU that the LDS allows (with up to 8 KB of a
// kernel's own).
template <typename T>
constexpr int waves_per_simd() { return T::NW / 4 * (T::LDS <= 73 * 1024 ? 2 : 1); }

// The loads of one side: per-lane offsets, the same for every tile, and the stage
// that comes next.
template <int B, bool KC, int N, bool WHOLE>
struct SideLoads {
  // Load i of a run lands 1024 i bytes on through its instruction offset, which
  // moves its memory address too: the per-lane offsets are less by as much,
  // and the descriptor starts kShift early to keep them positive.
  static constexpr uint32_t kShift = 1024 * (N < 4 ? N - 1 : 3);
  static constexpr int CPR = B / 8, RPI = 64 / CPR;     // RC: chunks of a row, rows of a load
  uint32_t voff[N];
  int32_t cut;             // KC: byte of load 0's chunk in its row (load 1's is the other half's)
  uint64_t at;
  int64_t step;            // bytes from one stage to the next
  int64_t ld2;             // bytes between rows
  int32_t extent, left;    // left: K from the next stage on
  int wave;

  // map: the memory row of a KC tile row.
  template <typename Map>
  __device__ __forceinline__ void init(int64_t ld, int w, int lane, Map&& map) {
    wave = w;
    ld2 = ld * 2;
    step = KC ? 128 : 64 * ld2;
    cut = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = KC ? 8 * (w * N + i) + (lane >> 3) : RPI * (w * N + i) + lane / CPR;
      const int c = KC ? (lane & 7) ^ swz_a64(r) : (lane % CPR) ^ swz_bn<B>(r);
      voff[i] = (uint32_t)((KC ? map(r) : r) * ld2) + c * 16u + kShift - 1024u * (i & 3);
      if (i == 0) cut = c * 16;
    }
  }
  __device__ __forceinline__ void tile(const Side& s) {
    extent = s.extent;
    left = s.k;
    at = reinterpret_cast<uint64_t>(s.base) - kShift;
  }
  // The descriptor of the next stage (of no memory past the last); *bytes: of a KC
  // row that are there.
  __device__ __forceinline__ i32x4 next(int32_t* bytes) {
    const int32_t k = min(left, 64);
    i32x4 d;
    d[0] = (int)(uint32_t)at;
    d[1] = (int)((at >> 32) & 0xffffu);
    d[2] = k > 0 ? (KC ? (int32_t)((extent - 1) * ld2) + 2 * k : (int32_t)((k - 1) * ld2) + 2 * extent) + (int32_t)kShift : 0;
    d[3] = 0x00020000;
    *bytes = 2 * k;
    at += step;
    left -= 64;
    return d;
  }
  __device__ __forceinline__ void load(const i32x4& d, int32_t bytes, const char* lds, int i) const {
    uint32_t v = voff[i];
    // consecutive loads' rows differ in bit 2 of their swizzle
    if constexpr (KC && !WHOLE) v = (cut ^ (64 * (i & 1))) < bytes ? v : 0x80000000u;
    lds_dma16_run<false>(d, v, 0u, lds + (wave * N + i) * 1024, i & 3);
  }
};

// A fragment of one side in a stage's half kk: 16 x 32 of a wave's T tiles, lane l
// with row l % 16 and K 8 (l / 16) .. + 7. STEP: rows (KC) between tiles.
template <int B, bool KC, int T, int STEP>
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
  static_assert(KC || ((T & (T - 1)) == 0 && STEP == 16), "the wave's columns start at a multiple of their number");
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
  // Read h of tile t.
  __device__ __forceinline__ void read(uint32_t (&at)[NA], int kk, int t, int h, int32_t move) {
    // a tile's own address moves to another stage buffer with its first read there
    if (!KC && h == 0) at[t] += move;
    if constexpr (KC) k = *(const lds_bf16x8*)(uintptr_t)(at[kk] + t * STEP * 128);
    else r[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(uintptr_t)(at[t] + h * 4 * B * 2 + kk * 32 * B * 2));
  }
  __device__ __forceinline__ bf16x8 get() const {
    if constexpr (KC) return k;
    else return __builtin_bit_cast(bf16x8, __builtin_shufflevector(r[0], r[1], 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// Nothing of the workgroup's LDS accesses before this is behind it; at most VM of
// a wave's memory accesses are on their way.
template <int VM>
__device__ __forceinline__ void product_barrier() {
  __builtin_amdgcn_s_waitcnt(waitcnt_imm(VM, 0));
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Steps, of a stage each, of a tile of k K: at least as many as are loaded ahead (the
// further ones are zeros), so that the loads are never more than a tile ahead.
template <typename T>
__device__ __forceinline__ int32_t product_steps(int32_t k) { return max((k + 63) / 64, T::AHEAD); }

#if defined(__HIP_DEVICE_COMPILE__)
// This workgroup's tiles one after the other. next(i, &work) gives its i-th, a
// struct with the Sides u and v and the number of steps (uniform; false: no
// more; also called one beyond); finish(work, acc) takes the fp32 sums, and may use LDS
// outside sm, T::LDS bytes, 1024-byte aligned. ldu, ldv: elements between
// memory rows; vmap: the memory row of a KC V tile row. STORES: how many memory accesses
// finish makes in every wave whatever the tile (each store of a TileMatrix counts, also
// of rows that are not there); 0: it is not known.
//
// A half's MFMAs go tile row by tile row of U: as soon as a row's are issued, its
// fragment's registers take the next half's. The last two rows and V have two
// sets, read first, so that every read of a stage is a good part of a half old at
// the barrier (whole second sets of U too would not fit beside a 256x256 tile's
// accumulators).
template <typename T, typename Work, int STORES, typename Next, typename VMap, typename Finish>
__device__ __forceinline__ void product_tiles(int64_t ldu, int64_t ldv, char* sm, int tid, Next&& next, VMap&& vmap,
                                              Finish&& finish) {
  constexpr int NS = T::NS, TM = T::TM, TN = T::TN;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / T::WGN, wn = wave % T::WGN;
  using FU = SideFrag<T::BM, T::UK, TM, T::UK ? 16 * T::WGM : 16>;
  using FV = SideFrag<T::BN, T::VK, TN, 16>;
  constexpr int SP = TM < 2 ? TM : 2, KEPT = TM - SP;    // rows of U with two sets, and with one
  Work cur, nxt;
  if (!next(0, &cur)) return;
  bool more = next(1, &nxt);
  FU fu[KEPT ? KEPT : 1], fs[2][SP];
  FV fv[2][TN];
  uint32_t ua[FU::NA], va[FV::NA];
  FU::addresses(sm + T::U_AT, T::row(wm, 0), lane, ua);
  FV::addresses(sm + T::V_AT, wn * T::WN, lane, va);
  SideLoads<T::BM, T::UK, T::NU, T::WHOLE> lu;
  SideLoads<T::BN, T::VK, T::NV, T::WHOLE> lv;
  lu.init(ldu, wave, lane, [](int r) { return r; });
  lv.init(ldv, wave, lane, vmap);
  lu.tile(cur.u);
  lv.tile(cur.v);
  int32_t to_load = cur.steps;         // stages of the tile being loaded
  int32_t loading = 0, reading = 0;              // stage buffers of the next load, of the last read

  f32x4 acc[TM][TN];
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  };
  clear();
  // 16-row tiles of the wave's with valid rows
  auto rows_of = [&](const Work& w) __attribute__((always_inline)) {
    return T::SKIP ? __builtin_amdgcn_readfirstlane((w.u.extent - 16 * wm + 16 * T::WGM - 1) / (16 * T::WGM)) : TM;
  };
  int32_t live = rows_of(cur), live_next = live;

  struct Stage {
    i32x4 du, dv;
    int32_t ku, kv;
    char *u, *v;
  };
  // The next stage, in three pieces that go between MFMAs.
  auto next_stage = [&](Stage& st, int piece) __attribute__((always_inline)) {
    if (piece == 0) {
      if (to_load == 0 && more) {      // on to the next tile's; without one, left is not positive any more
        lu.tile(nxt.u);
        lv.tile(nxt.v);
        to_load = nxt.steps;
      }
      --to_load;
    } else if (piece == 1) {
      st.du = lu.next(&st.ku);
      st.u = sm + T::U_AT + loading * T::U_BYTES;
    } else {
      st.dv = lv.next(&st.kv);
      st.v = sm + T::V_AT + loading * T::V_BYTES;
      loading = loading == NS - 1 ? 0 : loading + 1;
    }
  };
  auto load_one = [&](const Stage& st, int i) __attribute__((always_inline)) {
    if (i < T::NU) lu.load(st.du, st.ku, st.u, i);
    else lv.load(st.dv, st.kv, st.v, i - T::NU);
  };

  auto mfma_one = [&](int set, int mt, int nt) __attribute__((always_inline)) {
    const bf16x8 a = mt < KEPT ? fu[mt < KEPT ? mt : 0].get() : fs[set][mt < KEPT ? 0 : mt - KEPT].get();
    acc[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fv[set][nt].get(), a, acc[mt][nt], 0, 0, 0);
  };
  // Reads into the second sets: V's tiles and U's last rows, in this order.
  constexpr int kV = TN * FV::READS, kFirst = kV + SP * FU::READS;
  int32_t u_move = 0, v_move = 0;
  auto read_first = [&](int set, int kk, int i, bool move) __attribute__((always_inline)) {
    if (i < kV) fv[set][i / FV::READS].read(va, kk, i / FV::READS, i % FV::READS, move ? v_move : 0);
    else fs[set][(i - kV) / FU::READS].read(ua, kk, KEPT + (i - kV) / FU::READS, (i - kV) % FU::READS, move ? u_move : 0);
  };
  auto read_row = [&](int kk, int mt, bool move) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < FU::READS; ++h) fu[mt].read(ua, kk, mt, h, move ? u_move : 0);
  };
  // One half on set `set`; behind its MFMAs the reads of the next one (half kk at
  // the current addresses, moved before where it is in another buffer, of a tile with
  // `rows` 16-row tiles), `loads` loads of st and, with `plan`, the pieces of the next
  // stage to load.
  auto half = [&](int set, int kk, bool move, int rows, int loads, bool plan, Stage& st) __attribute__((always_inline)) {
    if constexpr (T::SKIP) {
      const int ops = kFirst + loads, per = (ops + TM - 1) / TM;
#pragma unroll
      for (int mt = 0; mt < TM; ++mt) {
        if (mt < live) {
#pragma unroll
          for (int nt = 0; nt < TN; ++nt) mfma_one(set, mt, nt);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < per; ++j) {
          const int i = mt * per + j;
          if (i < kFirst) read_first(set ^ 1, kk, i, move);
          else if (i < ops) load_one(st, i - kFirst);
        }
        if (mt < KEPT) {
          if constexpr (!T::UK) read_row(kk, mt, move);
          else if (mt < rows) read_row(kk, mt, move);
        }
        if (plan) {
#pragma unroll
          for (int i = 0; i < 3; ++i)
            if (mt == i * TM / 3) next_stage(st, i);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      constexpr int kMfma = TM * TN;
      const int all = kFirst + loads > kMfma ? kFirst + loads : kMfma;
#pragma unroll
      for (int i = 0; i < all; ++i) {
        if (i < kMfma) mfma_one(set, i / TN, i % TN);
        if (i < kFirst) read_first(set ^ 1, kk, i, move);
        else if (i < kFirst + loads) load_one(st, i - kFirst);
        if (i < kMfma && (i + 1) % TN == 0 && i / TN < KEPT) read_row(kk, i / TN, move);
        if (plan) {
#pragma unroll
          for (int j = 0; j < 3; ++j)
            if (i == (j + 1) * kMfma / 4) next_stage(st, j);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  Stage st;

#pragma unroll
  for (int j = 0; j < T::AHEAD; ++j) {
#pragma unroll
    for (int i = 0; i < 3; ++i) next_stage(st, i);
#pragma unroll
    for (int i = 0; i < T::NL; ++i) load_one(st, i);
  }
  // Every wave's part of a stage is there, and the loads of `after` later ones may be on their way.
  auto stage_barrier = [&](auto after) __attribute__((always_inline)) { product_barrier<decltype(after)::value * T::NL>(); };
  // The reads go on to the next stage buffer: a KC side's addresses at once, an RC
  // side's tiles as they are read.
  auto advance = [&]() __attribute__((always_inline)) {
    const int32_t by = reading == NS - 1 ? 1 - NS : 1;
    reading += by;
    u_move = by * T::U_BYTES;
    v_move = by * T::V_BYTES;
    if constexpr (T::UK) {
      ua[0] += u_move;
      ua[1] += u_move;
    }
    if constexpr (T::VK) {
      va[0] += v_move;
      va[1] += v_move;
    }
  };
  stage_barrier(std::integral_constant<int, T::AHEAD - 1>{});
#pragma unroll
  for (int i = 0; i < kFirst; ++i) read_first(0, 0, i, false);
#pragma unroll
  for (int i = 0; i < KEPT; ++i) read_row(0, i, false);

  bool fresh = false;
  for (int32_t i = 2;; ++i) {
    if (more) live_next = rows_of(nxt);
    // Steps; on entry set 0 holds the first half of one.
    for (int32_t s = cur.steps; s > 0; --s) {
      const int32_t rows = s > 1 ? live : live_next;      // of the step whose first half the second one reads
      half(0, 1, false, live, 0, true, st);
      // A wave's accesses finish in order: the first barrier after a tile's finish waits
      // for loads older than its stores, which may still be on their way (dW of 128
      // experts, 1536 x 2048 from 256 rows each: 394 -> 378 us).
      if (STORES && fresh) product_barrier<(T::AHEAD - 2) * T::NL + STORES>();
      else stage_barrier(std::integral_constant<int, T::AHEAD - 2>{});
      fresh = false;
      advance();
      half(1, 0, true, rows, T::NL, false, st);
    }
    finish(cur, acc);
    fresh = true;
    if (!more) break;
    cur = nxt;
    live = live_next;
    more = next(i, &nxt);
    clear();
  }
  // loads past the last stage write zeros to LDS: not after the workgroup's end
  __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, 0));
}
#endif

// The number of this workgroup's i-th tile. Rounds of gridDim.x tiles are dealt to the
// XCDs (workgroup mod 8) in runs of chunk (a divisor of a round's eighth), so that
// what runs on one XCD together shares operands in its L2; every other round backwards,
// so that where tiles get smaller from one to the next no workgroup has all the larger
// ones.
__device__ __forceinline__ int32_t dealt_tile(int i, uint32_t chunk) {
  const uint32_t b = i & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
  const uint32_t slot = b >> 3, run = __builtin_amdgcn_readfirstlane(slot / chunk);
  return (int32_t)(i * gridDim.x + (run * 8 + (b & 7)) * chunk + (slot - run * chunk));
}

// Tile `id` in a raster of `group` tile rows, column by column.
__device__ __forceinline__ void raster(int32_t id, int32_t tiles_m, int32_t tiles_n, int32_t group, int32_t* ti, int32_t* tj) {
  const int32_t per = group * tiles_n, r = __builtin_amdgcn_readfirstlane(id / per), first = r * group;
  const int32_t h = min(group, tiles_m - first), w = id - r * per;
  *tj = __builtin_amdgcn_readfirstlane(w / h);
  *ti = first + w - *tj * h;
}

// ---- storing a tile ----
// A lane holds row l % 16 and columns 4 (l / 16) .. + 3 of each 16x16 tile. Of two
// neighbouring ones, v_permlane16_swap_b32 hands lanes of even 16s the first's
// columns 4 (l / 16) .. + 7 and lanes of odd 16s the second's 4 (l / 16 - 1) .. + 7:
// 16 bytes of bf16 a lane, 64 contiguous bytes a row, without LDS. It is its own
// inverse.

// The column (in two tiles' 32) of a lane's eight.
__device__ __forceinline__ int pair_column(int lane) { return 16 * ((lane >> 4) & 1) + 8 * (lane >> 5); }

// A lane's eights of a wave's tiles in a bf16 matrix: rows < rows and columns < cols
// from `corner` on exist (at most 2^30 bytes of them); what lies past them reads as 0
// and is not stored. row0, col0: the lane's row and first column. NP pairs of 16x16
// tiles side by side, rows of them STEP apart. (Offsets and the bounds in a descriptor:
// a third of the vector instructions of 64-bit addresses and comparisons.)
template <int NP, int STEP>
struct TileMatrix {
  __amdgpu_buffer_rsrc_t memory;
  uint32_t at[NP];
  uint32_t step;
  __device__ __forceinline__ TileMatrix(const uint16_t* corner, int64_t ld, int32_t rows, int32_t cols, int32_t row0, int32_t col0) {
    const int32_t bytes = rows > 0 && cols > 0 ? (int32_t)((rows - 1) * ld + cols) * 2 : 0;
    memory = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(corner), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
    step = (uint32_t)(STEP * ld * 2);
#pragma unroll
    for (int i = 0; i < NP; ++i)
      at[i] = col0 + 32 * i < cols ? (uint32_t)(row0 * (int32_t)ld + col0 + 32 * i) * 2u : 0x80000000u;
  }
  __device__ __forceinline__ void store(int mt, int i, uint4 v) const {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(i32x4, v), memory, (int)(at[i] + mt * step), 0, 0);
  }
  __device__ __forceinline__ uint4 load(int mt, int i) const {
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(memory, (int)(at[i] + mt * step), 0, 0));
  }
};

__device__ __forceinline__ void swap16(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
// Four columns of each of two tiles -> eight columns of one.
__device__ __forceinline__ uint4 pair_up(uint2 a, uint2 b) {
  swap16(a.x, b.x);
  swap16(a.y, b.y);
  return make_uint4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ void pair_down(uint4 v, uint2* a, uint2* b) {
  *a = make_uint2(v.x, v.y);
  *b = make_uint2(v.z, v.w);
  swap16(a->x, b->x);
  swap16(a->y, b->y);
}

}  // namespace

}  // namespace ccl
