// A whole mixture-of-experts FFN layer for a few tokens (ccl_moe_decode):
//   route    p = softmax(logits) over the experts; the top_k largest, the
//            lowest expert first among equals; probabilities renormalised over
//            them where asked
//   up       h = act(s_e Wg x) * (s_e Wu x) for every (token, chosen expert)
//   down     y = sum over the chosen experts of p s'_e Wd h
//
// Bound by reading the chosen experts' weights once: a token's 2 operations
// per weight are far below what the matrix cores do per byte, so they do the
// products (v_mfma_f32_16x16x32_bf16, 16 weight rows by 16 tokens) even for one
// token, and the kernels are built around the weight stream:
//  * weights are read as they are stored (a checkpoint's output-major rows), 16
//    rows at a time, each lane 16 bytes, two loads covering a row's 128-byte
//    line; straight into registers, since no value is used twice;
//  * the K of a product is cut over the 8 waves of a workgroup, so that all of a
//    workgroup's rows are in flight at once, and summed through LDS in wave
//    order;
//  * tokens are gathered: an expert's product runs on the tokens that chose it
//    (16 at a time), rows of x and h coming from the caches.
// h crosses from the up to the down launch as bf16 pairs (rounded value and
// rounding error: 16 bits of the fp32 value), so that y is rounded once, at the
// end. Sums over K, over experts and the softmax are fp32, in a fixed order.
//
// Measured, us a call: one token, 8 of 128 experts of 2048 x 768 in bf16 (75 MB)
// 25 to 26: up 17, of which launch, routing and the sums about 6 and the weights 4.6
// TB/s; down 9, of 128 workgroups on 256 CUs; in fp8 19. 48 tokens over the same
// experts in fp8 (577 MB) 129, 4.5 TB/s: up 84, down 44, its ranges' sum 5; in bf16
// (1153 MB) 212, 5.4 TB/s.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "activation.hpp"
#include "kernels.hpp"

namespace ccl {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kRegs = kMoeMaxExperts / 64;        // logits of a token per lane

struct MoeParams {
  const uint16_t* x;
  const float* logits;
  const uint8_t* gate_up;
  const uint8_t* down;
  const float* gate_up_scale;   // per expert (null: 1)
  const float* down_scale;
  uint16_t* y;
  int32_t* ids;                 // caller's [tokens][top_k] (null: not wanted)
  float* probs;
  int32_t* ws_ids;              // the same in the workspace
  float* ws_probs;
  uint16_t* h;                  // [tokens * top_k][ffn / 8][8 values, 8 rests]
  float* part;                  // [splits][tokens][hidden] sums of the down product's ranges (null: one range)
  int64_t x_ld, logits_ld, y_ld;
  int64_t gu_stride, gu_ld, down_stride, down_ld;   // elements
  int32_t tokens, hidden, ffn, experts, top_k, act, normalize;
  int32_t list;                 // up: workgroups go by chosen (token, slot), not by expert
  int32_t tiles;                // up: 16-row tiles of ffn; down: of hidden
  int32_t group, groups;        // up: tiles per workgroup, workgroups per expert; down: tile groups
  int32_t splits;               // down: ranges of the (expert, K) steps
};

// Logits in an order-preserving form, 0 for what is never chosen (-inf, NaN).
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);      // -0 equals 0
  const uint32_t k = (u >> 31) ? ~u : u | 0x80000000u;
  return v > -__builtin_inff() ? k : 0u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k >> 31) ? k & 0x7fffffffu : ~k);
}

template <int CTRL>
__device__ __forceinline__ uint32_t max_step(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
  return v > o ? v : o;
}
// Maximum over the wave, in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max_step<0x111>(v);       // row_shr:1, 2, 4, 8
  v = max_step<0x112>(v);
  v = max_step<0x114>(v);
  v = max_step<0x118>(v);
  v = max_step<0x142>(v);       // row_bcast:15
  v = max_step<0x143>(v);       // row_bcast:31
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) v += __shfl_xor(v, x);
  return v;
}

// exp(v - top), 1 where they are equal (infinite ones too). The rounding of
// (v - top) log2 e, which grows with the distance, is carried as a factor.
__device__ __forceinline__ float exp_below(float v, float top) {
  constexpr float kRest = 1.92596299e-8f;           // log2 e - kLog2e
  if (v == top) return 1.f;
  const float d = v - top, e = d * kLog2e;
  const float rest = __builtin_fmaf(d, kRest, __builtin_fmaf(d, kLog2e, -e));
  // past the range of exp2 (d of -inf too) the rest does not count
  return e < -150.f ? 0.f : __builtin_amdgcn_exp2f(e) * __builtin_fmaf(rest, 0.693147181f, 1.f);
}

// One wave routes one token: ids and probabilities of its top_k slots (id -1,
// probability 0 where no expert is left) in lanes 0 .. top_k - 1.
__device__ __forceinline__ void route_token(const MoeParams& p, int t, int lane, int32_t* id_out, float* prob_out) {
  uint32_t key[kRegs];
  float all = 0.f;
  const float* row = p.logits + t * p.logits_ld;
  uint32_t best = 0;
#pragma unroll
  for (int r = 0; r < kRegs; ++r) {
    key[r] = 0;
    if (64 * r < p.experts) {
      const int e = 64 * r + lane;
      if (e < p.experts) key[r] = order_key(row[e]);
      best = best > key[r] ? best : key[r];
    }
  }
  const uint32_t first = wave_max(best);
  const float top = key_value(first);
  if (!p.normalize) {
#pragma unroll
    for (int r = 0; r < kRegs; ++r)
      if (key[r]) all += exp_below(key_value(key[r]), top);
    all = wave_sum(all);
  }
  int32_t id = -1;
  float w = 0.f, sum = 0.f;
  uint32_t m = first;
  for (int j = 0; j < p.top_k; ++j) {
    if (j) {
      best = 0;
#pragma unroll
      for (int r = 0; r < kRegs; ++r)
        if (64 * r < p.experts) best = best > key[r] ? best : key[r];
      m = wave_max(best);
    }
    if (m == 0) break;
    bool found = false;
#pragma unroll
    for (int r = 0; r < kRegs; ++r) {
      if (64 * r >= p.experts || found) break;
      const uint64_t hit = __ballot(key[r] == m);
      if (hit) {
        found = true;
        const int l = __builtin_ctzll(hit);
        const float e = exp_below(key_value(m), top);
        sum += e;
        if (lane == j) {
          id = 64 * r + l;
          w = e;
        }
        if (lane == l) key[r] = 0;
      }
    }
  }
  const float total = p.normalize ? sum : all;
  *id_out = id;
  *prob_out = id >= 0 ? w / total : 0.f;
}

__device__ __forceinline__ void put_route(const MoeParams& p, int t, int lane, int32_t id, float prob) {
  if (lane >= p.top_k) return;
  const int i = t * p.top_k + lane;
  p.ws_ids[i] = id;
  p.ws_probs[i] = prob;
  if (p.ids) p.ids[i] = id;
  if (p.probs) p.probs[i] = prob;
}

// Eight consecutive weights as bf16: what is loaded, or half of 16 fp8 values
// (exact: E4M3 fits in bf16).
// The empty asm keeps the conversion where its product is: hoisted out of a loop
// over token tiles, the converted weights took twice the registers and spilled.
__device__ __forceinline__ bf16x8 from_fp8(uint32_t a, uint32_t b) {
  asm volatile("" : "+v"(a), "+v"(b));
  const bf16x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false);
  const bf16x2 v1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
  const bf16x2 v2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false);
  const bf16x2 v3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
  return bf16x8{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
}

// A tile of 16 weight rows, read through a buffer descriptor: 16 bytes of a row
// are kPer values, a 128-byte line 8 such chunks, of which lane group g = lane /
// 16 takes g and g + 4. A chunk feeds kPer / 8 MFMAs, the v-th with its values
// 8 v .. 8 v + 7 (the K order inside an MFMA is free as long as both operands
// share it). Chunks past the row's end read as zeros.
typedef int i32x4 __attribute__((ext_vector_type(4)));

template <bool FP8>
struct Weights {
  static constexpr int kPer = FP8 ? 16 : 8;
  static constexpr int kLine = 8 * kPer;
  static constexpr int kMfma = kPer / 8;
  static constexpr uint32_t kNone = 0x80000000u;  // an offset past every tile
  // Lane offsets of the two chunks in a whole line and in the row's last.
  // Scalars, not arrays: an array that lambdas capture stays in memory.
  uint32_t v0, v1, end0, end1;
  int last;                     // the row's last line
  __device__ __forceinline__ Weights(int64_t ld, int K, int lane) {
    const int r = lane & 15, g = lane >> 4;
    last = (K - 1) / kLine;
    v0 = (uint32_t)(r * ld * (FP8 ? 1 : 2)) + 16u * g;
    v1 = v0 + 64u;
    end0 = last * kLine + g * kPer < K ? v0 : kNone;
    end1 = last * kLine + (g + 4) * kPer < K ? v1 : kNone;
  }
  // Chunk c of line l of the tile at `rows` (16 rows of ld).
  __device__ __forceinline__ uint4 load(__amdgpu_buffer_rsrc_t rows, int l, int c) const {
    const uint32_t v = l < last ? (c ? v1 : v0) : l == last ? (c ? end1 : end0) : kNone;
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rows, (int)v, l * 128, 0));
  }
  // Lane offsets of rows of x or h beside the weights': `bytes` of a row for each
  // weight value.
  __device__ __forceinline__ uint32_t beside(uint32_t row, int l, int c, int bytes) const {
    const uint32_t v = row + (c ? 4 * kPer * bytes : 0);
    return l < last || (c ? end1 : end0) != kNone ? v : kNone;
  }
  __device__ static __forceinline__ __amdgpu_buffer_rsrc_t tile(const uint8_t* rows, int64_t ld) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(rows), 0, (int)(16 * ld * (FP8 ? 1 : 2)), 0x00020000);
  }
  __device__ static __forceinline__ bf16x8 frag(uint4 w, int v) {
    if constexpr (FP8) return v == 0 ? from_fp8(w.x, w.y) : from_fp8(w.z, w.w);
    else return __builtin_bit_cast(bf16x8, w);
  }
};

__device__ __forceinline__ bf16x8 load8(__amdgpu_buffer_rsrc_t b, uint32_t v, int s) {
  return __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(b, (int)v, s, 0));
}

// A barrier that waits for the wave's LDS accesses but not for its loads, which
// may be the next step's weights.
__device__ __forceinline__ void staged_sync() {
  __builtin_amdgcn_s_waitcnt(0xc07f);               // lgkmcnt(0)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The up launch: one workgroup per expert and group of 16-row tiles (of gate
// and of up). The group is a stream of (tile, K chunk) steps: a step's weights
// are loaded behind the products of the step before, ahead of its sums. A wave
// keeps its x rows in registers where its share of K is one chunk. STREAM: a
// workgroup takes several tiles and may use 256 registers a lane, for the next
// step's weights in flight during this one's sums: 148 in bf16, where one workgroup
// has a CU to itself, 113 in fp8, where two share it. Otherwise a workgroup has one
// tile and at most 128 registers, and two share a CU.
template <bool FP8, bool STREAM>
__global__ void __launch_bounds__(kThreads, STREAM ? 2 : 4) moe_up_kernel(MoeParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  using W = Weights<FP8>;
  __shared__ int32_t s_ids[kMoeMaxExperts];       // list: chosen experts of all slots
  __shared__ int32_t s_entry[kMoeMaxTokens];      // the expert's slots (token * top_k + slot)
  __shared__ int32_t s_slot[kMoeMaxTokens];       // by expert: a token's slot (-1: not chosen)
  __shared__ int32_t s_n;
  extern __shared__ __attribute__((aligned(16))) float s_red[];   // [gate, up][wave][token slot][16]
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int slots = p.tokens * p.top_k;
  int expert, part;
  if (p.list) {
    const int slot = blockIdx.x / p.groups;
    part = blockIdx.x - slot * p.groups;
    for (int t = wave; t < p.tokens; t += kWaves) {
      int32_t id;
      float prob;
      route_token(p, t, lane, &id, &prob);
      if (lane < p.top_k) s_ids[t * p.top_k + lane] = id;
      if (blockIdx.x == 0) put_route(p, t, lane, id, prob);
    }
    if (p.tokens == 1 && threadIdx.x == 0) {      // one token's experts are distinct
      s_entry[0] = slot;
      s_n = 1;
    }
    __syncthreads();
    expert = s_ids[slot];
    if (expert < 0) return;
    if (wave == 0 && p.tokens > 1) {
      // The first slot of an expert does its work for all of them.
      int n = 0;
      bool first = true;
      for (int c = 0; c < slots; c += 64) {
        const bool hit = c + lane < slots && s_ids[c + lane] == expert;
        const uint64_t mask = __ballot(hit);
        if (n == 0 && mask && c + __builtin_ctzll(mask) < slot) first = false;
        if (hit) s_entry[n + __builtin_popcountll(mask & ((1ull << lane) - 1))] = c + lane;
        n += __builtin_popcountll(mask);
      }
      if (lane == 0) s_n = first ? n : 0;
    }
    if (p.tokens > 1) __syncthreads();
  } else {
    const int routers = (p.tokens + kWaves - 1) / kWaves;
    if ((int)blockIdx.x < routers) {
      const int t = blockIdx.x * kWaves + wave;
      if (t < p.tokens) {
        int32_t id;
        float prob;
        route_token(p, t, lane, &id, &prob);
        put_route(p, t, lane, id, prob);
      }
      return;
    }
    expert = (blockIdx.x - routers) / p.groups;
    part = blockIdx.x - routers - expert * p.groups;
    // The expert's rank among a token's logits is its slot. A wave ranks its
    // tokens together, so that their logits are in flight together.
    constexpr int kPer = kMoeMaxTokens / kWaves;
    uint32_t mine[kPer];
    int rank[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int t = wave + kWaves * i;
      mine[i] = t < p.tokens ? __float_as_uint(p.logits[t * p.logits_ld + expert]) : 0u;
      rank[i] = 0;
    }
    for (int e0 = 0; e0 < p.experts; e0 += 64) {
      const int e = e0 + lane;
      float v[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int t = wave + kWaves * i;
        v[i] = t < p.tokens && e < p.experts ? p.logits[t * p.logits_ld + e] : -__builtin_inff();
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const uint32_t k = order_key(v[i]), m = order_key(__uint_as_float(mine[i]));
        rank[i] += __builtin_popcountll(__ballot(k > m || (k == m && e < expert)));
      }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int t = wave + kWaves * i;
      if (lane == 0 && t < p.tokens)
        s_slot[t] = order_key(__uint_as_float(mine[i])) && rank[i] < p.top_k ? rank[i] : -1;
    }
    __syncthreads();
    if (wave == 0) {
      const int s = lane < p.tokens ? s_slot[lane] : -1;
      const uint64_t mask = __ballot(s >= 0);
      if (s >= 0) s_entry[__builtin_popcountll(mask & ((1ull << lane) - 1))] = lane * p.top_k + s;
      if (lane == 0) s_n = __builtin_popcountll(mask);
    }
    __syncthreads();
  }
  const int n = __builtin_amdgcn_readfirstlane(s_n);
  if (n == 0) return;
  expert = __builtin_amdgcn_readfirstlane(expert);
  part = __builtin_amdgcn_readfirstlane(part);

  const int K = p.hidden, F = p.ffn;
  const int r = lane & 15, g = lane >> 4;
  const int64_t esize = FP8 ? 1 : 2;
  const int tile0 = STREAM ? part * p.group : part, tile1 = STREAM ? min(p.tiles, tile0 + p.group) : tile0 + 1;
  const W weights(p.gu_ld, K, lane);
  constexpr int kLines = FP8 ? 2 : 4;                       // lines of a chunk
  const int lines = weights.last + 1;
  const int per = (lines + kWaves - 1) / kWaves;
  const int first = min(lines, wave * per), last = min(lines, first + per);
  const int chunks = (per + kLines - 1) / kLines;           // the same for every wave
  const int mts = (n + 15) / 16, rows = 16 * mts;
  const uint8_t* gate = p.gate_up + expert * p.gu_stride * esize;
  const uint8_t* up = gate + F * p.gu_ld * esize;

  // Token slots past the last read the last one's row: their columns of the
  // products are not used.
  const auto xb = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(p.x), 0,
                                                    (int)(((p.tokens - 1) * p.x_ld + K) * 2), 0x00020000);
  const auto x_row = [&](int mt) {
    return (uint32_t)((s_entry[min(16 * mt + r, n - 1)] / p.top_k * p.x_ld + g * W::kPer) * 2);
  };
  bf16x8 fx[kLines][2][W::kMfma];
  const auto load_x = [&](uint32_t row, int l0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kLines; ++i) {
      const int l = min(l0 + i, weights.last);
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int v = 0; v < W::kMfma; ++v)
          fx[i][c][v] = load8(xb, weights.beside(row, l, c, 2) + 16 * v, l * W::kLine * 2);
    }
  };
  uint4 wg[kLines][2], wu[kLines][2];
  const auto load_w = [&](int tile, int l0) __attribute__((always_inline)) {
    const auto tg = W::tile(gate + 16 * tile * p.gu_ld * esize, p.gu_ld);
    const auto tu = W::tile(up + 16 * tile * p.gu_ld * esize, p.gu_ld);
#pragma unroll
    for (int i = 0; i < kLines; ++i) {
      const int l = l0 + i < last ? l0 + i : lines;         // past the wave's share: nothing is read
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        wg[i][c] = weights.load(tg, l, c);
        wu[i][c] = weights.load(tu, l, c);
      }
    }
  };
  const uint32_t row0 = x_row(0);
  if (chunks == 1) load_x(row0, first);
  load_w(tile0, first);
  const float scale = p.gate_up_scale ? p.gate_up_scale[expert] : 1.f;
  const ActCoef ak = act_coef(p.act);
  int tile = tile0;
  do {
    for (int ch = 0; ch < chunks; ++ch) {
      const int l0 = first + ch * kLines;
      for (int mt = mts - 1; mt >= 0; --mt) {               // the first tile last: its x stays
        if (chunks > 1 || mts > 1) load_x(mt ? x_row(mt) : row0, l0);
        f32x4 ag{0.f, 0.f, 0.f, 0.f}, au = ag;
#pragma unroll
        for (int i = 0; i < kLines; ++i) {
          if (l0 + i >= last) break;
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int v = 0; v < W::kMfma; ++v) {
              ag = __builtin_amdgcn_mfma_f32_16x16x32_bf16(W::frag(wg[i][c], v), fx[i][c][v], ag, 0, 0, 0);
              au = __builtin_amdgcn_mfma_f32_16x16x32_bf16(W::frag(wu[i][c], v), fx[i][c][v], au, 0, 0, 0);
            }
        }
        // Lane l holds weight rows 4 (l / 16) .. + 3 for the token of slot l % 16.
        f32x4* sg = reinterpret_cast<f32x4*>(s_red + (wave * rows + 16 * mt + r) * 16 + 4 * g);
        f32x4* su = sg + kWaves * rows * 4;
        if (ch) {
          ag += *sg;
          au += *su;
        }
        *sg = ag;
        *su = au;
      }
      if (ch + 1 < chunks) load_w(tile, l0 + kLines);
      else if (STREAM && tile + 1 < tile1) load_w(tile + 1, first);
    }
    staged_sync();
    for (int at = threadIdx.x; at < n * 16; at += kThreads) {
      const int slot = at >> 4, f = 16 * tile + (at & 15);
      float zg = 0.f, zu = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        zg += s_red[(w * rows + slot) * 16 + (at & 15)];
        zu += s_red[((kWaves + w) * rows + slot) * 16 + (at & 15)];
      }
      float v = 0.f;
      with_act(p.act, [&](auto cls) { v = act_value<decltype(cls)::value>(ak, zg * scale); });
      v *= zu * scale;
      const __bf16 hi = (__bf16)v;
      const float rest = __builtin_fabsf((float)hi) < __builtin_inff() ? v - (float)hi : 0.f;
      const __bf16 lo = (__bf16)rest;
      uint16_t* h = p.h + (int64_t)s_entry[slot] * F * 2 + f / 8 * 16 + f % 8;
      h[0] = __builtin_bit_cast(uint16_t, hi);
      h[8] = __builtin_bit_cast(uint16_t, lo);
    }
    if (STREAM && tile + 1 < tile1) staged_sync();
  } while (STREAM && ++tile < tile1);
#endif
}

// The down launch: one workgroup per NT tiles of 16 rows of the down weights
// (columns of y) and range of the (expert, K line) steps of the chosen
// experts; the steps of a range are cut over the waves. A wave's stream is cut
// into units of up to kLines lines of one expert; a unit's weights are loaded behind
// the loads of the h rows of the unit before, one unit ahead of its products,
// which are added to the wave's own y in LDS, at the rows of the unit's tokens.
// Several tiles share the loads of h: with one, an fp8 layer's h took four times
// the weights' load instructions (48 tokens, 128 experts of 2048 x 768: 92 us).
template <bool FP8, int NT>
__global__ void __launch_bounds__(kThreads, 2) moe_down_kernel(MoeParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  using W = Weights<FP8>;
  constexpr int COLS = 16 * NT;
  constexpr int kSlots = kMoeMaxTokens * kMoeMaxTopK;
  __shared__ int32_t s_list[kSlots];              // slots by expert
  __shared__ float s_probs[kSlots];               // times the expert's scale
  __shared__ int32_t s_used[kMoeMaxExperts];      // experts chosen at all, ascending
  __shared__ int32_t s_count[kMoeMaxExperts], s_start[kMoeMaxExperts];
  __shared__ int32_t s_total;
  extern __shared__ __attribute__((aligned(16))) float s_y[];   // [wave][token][COLS]
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int slots = p.tokens * p.top_k;
  const int group = blockIdx.x % p.groups, split = blockIdx.x / p.groups;
  for (int i = threadIdx.x; i < kWaves * p.tokens * COLS / 4; i += kThreads)
    reinterpret_cast<f32x4*>(s_y)[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (p.tokens == 1) {
    // Its experts are distinct: in the order of their slots, without counting.
    if (wave == 0) {
      const int id = lane < slots ? p.ws_ids[lane] : -1;
      const uint64_t mask = __ballot(id >= 0);
      if (id >= 0) {
        const int at = __builtin_popcountll(mask & ((1ull << lane) - 1));
        s_probs[lane] = p.ws_probs[lane] * (p.down_scale ? p.down_scale[id] : 1.f);
        s_used[at] = id;
        s_count[id] = 1;
        s_start[id] = at;
        s_list[at] = lane;
      }
      if (lane == 0) s_total = __builtin_popcountll(mask);
    }
    __syncthreads();
  } else {
    int32_t my_id[2], my_rank[2];                   // kSlots / kThreads slots per thread
    for (int e = threadIdx.x; e < p.experts; e += kThreads) s_count[e] = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int i = threadIdx.x + j * kThreads;
      my_id[j] = i < slots ? p.ws_ids[i] : -1;
      if (my_id[j] >= 0) s_probs[i] = p.ws_probs[i] * (p.down_scale ? p.down_scale[my_id[j]] : 1.f);
    }
    __syncthreads();
    // The order of an expert's slots in its list is free: it places rows of a
    // product, whose sums do not mix rows.
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (my_id[j] >= 0) my_rank[j] = atomicAdd(&s_count[my_id[j]], 1);
    __syncthreads();
    if (wave == 0) {
      int used = 0, start = 0;
      for (int e0 = 0; e0 < p.experts; e0 += 64) {
        const int c = e0 + lane < p.experts ? s_count[e0 + lane] : 0;
        const uint64_t mask = __ballot(c > 0);
        if (c > 0) s_used[used + __builtin_popcountll(mask & ((1ull << lane) - 1))] = e0 + lane;
        used += __builtin_popcountll(mask);
        int sum = c;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) {
          const int o = __shfl_up(sum, x);
          if (lane >= x) sum += o;
        }
        if (e0 + lane < p.experts) s_start[e0 + lane] = start + sum - c;
        start += __shfl(sum, 63);
      }
      if (lane == 0) s_total = used;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (my_id[j] >= 0) s_list[s_start[my_id[j]] + my_rank[j]] = threadIdx.x + j * kThreads;
    __syncthreads();
  }

  const int K = p.ffn, D = p.hidden;
  const int r = lane & 15, g = lane >> 4;
  const int64_t esize = FP8 ? 1 : 2;
  const W weights(p.down_ld, K, lane);
  constexpr int kLines = NT == 1 ? 4 : 2;                   // lines of a unit
  const int lines = weights.last + 1;
  const int total = __builtin_amdgcn_readfirstlane(s_total) * lines;
  const int parts = p.splits * kWaves, part = split * kWaves + wave;
  const int begin = __builtin_amdgcn_readfirstlane((int)((int64_t)total * part / parts));
  const int end = __builtin_amdgcn_readfirstlane((int)((int64_t)total * (part + 1) / parts));
  struct Unit {
    int index, expert, l0, l1;  // of the used experts; lines l0 .. l1 - 1
  };
  const auto unit_of = [&](int index, int l0, int left) __attribute__((always_inline)) {
    return Unit{index, __builtin_amdgcn_readfirstlane(s_used[index]), l0, min(min(lines, l0 + kLines), l0 + left)};
  };
  const auto after = [&](const Unit& t, int left) __attribute__((always_inline)) {
    return t.l1 == lines ? unit_of(t.index + 1, 0, left) : unit_of(t.index, t.l1, left);
  };
  const auto load_w = [&](const Unit& t, uint4 (&w)[NT][kLines][2]) __attribute__((always_inline)) {
    const uint8_t* base = p.down + t.expert * p.down_stride * esize;
#pragma unroll
    for (int m = 0; m < NT; ++m) {
      // tiles past the last read the last one, and are not stored
      const auto rows = W::tile(base + 16 * min(group * NT + m, p.tiles - 1) * p.down_ld * esize, p.down_ld);
#pragma unroll
      for (int i = 0; i < kLines; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) w[m][i][c] = weights.load(rows, t.l0 + i < t.l1 ? t.l0 + i : lines, c);
    }
  };
  const auto hb = __builtin_amdgcn_make_buffer_rsrc(p.h, 0, slots * K * 4, 0x00020000);
  const auto run = [&](const Unit& t, const uint4 (&w)[NT][kLines][2], auto&& between) __attribute__((always_inline)) {
    const int n = __builtin_amdgcn_readfirstlane(s_count[t.expert]), start = __builtin_amdgcn_readfirstlane(s_start[t.expert]);
    // Eight slots at a time: columns 0 .. 7 of the products are their values,
    // 8 .. 15 their rests, added at the end.
    for (int m0 = 0; m0 < n; m0 += 8) {
      // slots past the last: the last one's row, and its products are dropped
      const int slot = s_list[start + min(m0 + (r & 7), n - 1)];
      const uint32_t row = (uint32_t)(slot * K + g * W::kPer) * 4u + (r & 8 ? 16u : 0u);
      bf16x8 h[kLines][2][W::kMfma];
#pragma unroll
      for (int i = 0; i < kLines; ++i) {
        const int l = min(t.l0 + i, weights.last);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int v = 0; v < W::kMfma; ++v)
            h[i][c][v] = load8(hb, weights.beside(row, l, c, 4) + 32 * v, l * W::kLine * 4);
      }
      if (m0 == 0) between();
      f32x4 acc[NT];
#pragma unroll
      for (int m = 0; m < NT; ++m) acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kLines; ++i) {
        if (t.l0 + i >= t.l1) break;
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int v = 0; v < W::kMfma; ++v)
#pragma unroll
            for (int m = 0; m < NT; ++m)
              acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(W::frag(w[m][i][c], v), h[i][c][v], acc[m], 0, 0, 0);
      }
#pragma unroll
      for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[m][j] += __shfl_xor(acc[m][j], 8);
      if (r < 8 && m0 + r < n) {
        float* y = s_y + (wave * p.tokens + slot / p.top_k) * COLS + 4 * g;
        const float weight = s_probs[slot];
#pragma unroll
        for (int m = 0; m < NT; ++m) *reinterpret_cast<f32x4*>(y + 16 * m) += acc[m] * weight;
      }
    }
  };
  uint4 wa[NT][kLines][2], wb[NT][kLines][2];
  if (begin < end) {
    int left = end - begin;
    Unit t = unit_of(begin / lines, begin % lines, left), u = t;
    load_w(t, wa);
    while (true) {
      // two units a round, so that the buffers' names are fixed
      left -= t.l1 - t.l0;
      if (left > 0) u = after(t, left);
      run(t, wa, [&]() __attribute__((always_inline)) { if (left > 0) load_w(u, wb); });
      if (left <= 0) break;
      left -= u.l1 - u.l0;
      if (left > 0) t = after(u, left);
      run(u, wb, [&]() __attribute__((always_inline)) { if (left > 0) load_w(t, wa); });
      if (left <= 0) break;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < p.tokens * COLS; i += kThreads) {
    const int t = i / COLS, c = group * COLS + i % COLS;
    if (c >= D) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += s_y[w * p.tokens * COLS + i];
    if (p.part) p.part[((int64_t)split * p.tokens + t) * D + c] = v;
    else p.y[t * p.y_ld + c] = __builtin_bit_cast(uint16_t, (__bf16)v);
  }
#endif
}

// The sum of the down product's ranges, in order, four columns a thread.
__global__ void __launch_bounds__(256) moe_sum_kernel(MoeParams p) {
  const int64_t n = (int64_t)p.tokens * p.hidden / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < p.splits; ++s) v += reinterpret_cast<const f32x4*>(p.part)[s * n + i];
  const int64_t t = 4 * i / p.hidden;
  uint16_t* y = p.y + t * p.y_ld + (4 * i - t * p.hidden);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __bf16 b = (__bf16)v[j];
    y[j] = __builtin_bit_cast(uint16_t, b);
  }
}

}  // namespace

hipError_t launch_moe(const MoeShape& s, const MoeCall& c, void* ws, hipStream_t stream) {
  const MoeForm f = moe_form(s, c.tokens);
  char* base = static_cast<char*>(ws);
  MoeParams p;
  p.x = static_cast<const uint16_t*>(c.x);
  p.logits = c.logits;
  p.gate_up = static_cast<const uint8_t*>(c.gate_up);
  p.down = static_cast<const uint8_t*>(c.down);
  p.gate_up_scale = c.gate_up_scale;
  p.down_scale = c.down_scale;
  p.y = static_cast<uint16_t*>(c.y);
  p.ids = c.ids;
  p.probs = c.probs;
  p.ws_ids = reinterpret_cast<int32_t*>(base);
  p.ws_probs = reinterpret_cast<float*>(base + f.probs_at);
  p.h = reinterpret_cast<uint16_t*>(base + f.h_at);
  p.part = f.splits > 1 ? reinterpret_cast<float*>(base + f.part_at) : nullptr;
  p.x_ld = c.x_ld;
  p.logits_ld = c.logits_ld;
  p.y_ld = c.y_ld;
  p.gu_stride = s.gu_stride;
  p.gu_ld = s.gu_ld;
  p.down_stride = s.down_stride;
  p.down_ld = s.down_ld;
  p.tokens = (int32_t)c.tokens;
  p.hidden = (int32_t)s.hidden;
  p.ffn = (int32_t)s.ffn;
  p.experts = s.experts;
  p.top_k = s.top_k;
  p.act = s.act;
  p.normalize = s.normalize ? 1 : 0;
  p.list = f.list ? 1 : 0;
  p.tiles = f.up_tiles;
  p.group = f.up_group;
  p.groups = (f.up_tiles + f.up_group - 1) / f.up_group;
  p.splits = f.splits;
  const unsigned red = (unsigned)((c.tokens + 15) / 16 * 16 * 2 * kWaves * 16 * sizeof(float));
  const dim3 up((unsigned)f.up_workgroups), block(kThreads);
  if (s.fp8 && f.up_group > 1) hipLaunchKernelGGL((moe_up_kernel<true, true>), up, block, red, stream, p);
  else if (s.fp8) hipLaunchKernelGGL((moe_up_kernel<true, false>), up, block, red, stream, p);
  else if (f.up_group > 1) hipLaunchKernelGGL((moe_up_kernel<false, true>), up, block, red, stream, p);
  else hipLaunchKernelGGL((moe_up_kernel<false, false>), up, block, red, stream, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  p.tiles = f.down_tiles;
  p.groups = f.down_groups;
  const dim3 down((unsigned)(f.down_groups * f.splits));
  const unsigned sums = (unsigned)(kWaves * c.tokens * 16 * f.down_nt * sizeof(float));
  if (f.down_nt == 1) {
    if (s.fp8) hipLaunchKernelGGL((moe_down_kernel<true, 1>), down, block, sums, stream, p);
    else hipLaunchKernelGGL((moe_down_kernel<false, 1>), down, block, sums, stream, p);
  } else {
    if (s.fp8) hipLaunchKernelGGL((moe_down_kernel<true, kMoeDownTiles>), down, block, sums, stream, p);
    else hipLaunchKernelGGL((moe_down_kernel<false, kMoeDownTiles>), down, block, sums, stream, p);
  }
  e = hipGetLastError();
  if (e != hipSuccess || f.splits == 1) return e;
  hipLaunchKernelGGL(moe_sum_kernel, dim3((unsigned)((c.tokens * s.hidden / 4 + 255) / 256)), dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace ccl
