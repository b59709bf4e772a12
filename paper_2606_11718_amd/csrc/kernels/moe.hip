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
constexpr int kTiles = kMoeMaxTokens / 16;        // 16-token tiles of an expert

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
      for (int r = 0; r < kRegs; ++r) best = best > key[r] ? best : key[r];
      m = wave_max(best);
    }
    if (m == 0) break;
    bool found = false;
#pragma unroll
    for (int r = 0; r < kRegs; ++r) {
      const uint64_t hit = __ballot(key[r] == m);
      if (!found && hit) {
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
__device__ __forceinline__ bf16x8 from_fp8(uint32_t a, uint32_t b) {
  const bf16x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false);
  const bf16x2 v1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
  const bf16x2 v2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false);
  const bf16x2 v3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
  return bf16x8{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
}

// 16 bytes of a weight row are kPer values; a 128-byte line is 8 such chunks.
// Lane group g = lane / 16 takes chunks g and g + 4 of a line. A chunk feeds
// kPer / 8 MFMAs, the v-th with its values 8 v .. 8 v + 7 (the K order inside an
// MFMA is free as long as both operands share it).
template <bool FP8>
struct Weights {
  static constexpr int kPer = FP8 ? 16 : 8;
  static constexpr int kLine = 8 * kPer;
  static constexpr int kMfma = kPer / 8;
  __device__ static __forceinline__ uint4 load(const uint8_t* row, int k, int K) {
    return k < K ? *reinterpret_cast<const uint4*>(row + (int64_t)k * (FP8 ? 1 : 2)) : make_uint4(0, 0, 0, 0);
  }
  __device__ static __forceinline__ bf16x8 frag(uint4 w, int v) {
    if constexpr (FP8) return v == 0 ? from_fp8(w.x, w.y) : from_fp8(w.z, w.w);
    else return __builtin_bit_cast(bf16x8, w);
  }
};

__device__ __forceinline__ bf16x8 zero8() { return __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0)); }

// The up launch: one workgroup per (expert, 16 rows of gate and of up).
template <bool FP8>
__global__ void __launch_bounds__(kThreads, 4) moe_up_kernel(MoeParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  using W = Weights<FP8>;
  __shared__ int32_t s_ids[kMoeMaxExperts];       // list: chosen experts of all slots
  __shared__ int32_t s_entry[kMoeMaxTokens];      // the expert's slots (token * top_k + slot)
  __shared__ int32_t s_slot[kMoeMaxTokens];       // by expert: a token's slot (-1: not chosen)
  __shared__ int32_t s_n;
  __shared__ __attribute__((aligned(16))) float s_red[2][kWaves][16][16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int slots = p.tokens * p.top_k;
  int expert, tile;
  if (p.list) {
    const int slot = blockIdx.x / p.tiles;
    tile = blockIdx.x - slot * p.tiles;
    for (int t = wave; t < p.tokens; t += kWaves) {
      int32_t id;
      float prob;
      route_token(p, t, lane, &id, &prob);
      if (lane < p.top_k) s_ids[t * p.top_k + lane] = id;
      if (blockIdx.x == 0) put_route(p, t, lane, id, prob);
    }
    __syncthreads();
    expert = s_ids[slot];
    if (expert < 0) return;
    if (wave == 0) {
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
    __syncthreads();
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
    expert = (blockIdx.x - routers) / p.tiles;
    tile = blockIdx.x - routers - expert * p.tiles;
    // The expert's rank among a token's logits is its slot.
    for (int t = wave; t < p.tokens; t += kWaves) {
      const float* row = p.logits + t * p.logits_ld;
      const uint32_t mine = order_key(row[expert]);
      int rank = 0;
      for (int e0 = 0; e0 < p.experts; e0 += 64) {
        const int e = e0 + lane;
        const uint32_t k = e < p.experts ? order_key(row[e]) : 0u;
        rank += __builtin_popcountll(__ballot(k > mine || (k == mine && e < expert)));
      }
      if (lane == 0) s_slot[t] = mine && rank < p.top_k ? rank : -1;
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

  const int K = p.hidden, F = p.ffn;
  const int f0 = 16 * tile, r = lane & 15, g = lane >> 4;
  const int frow = min(f0 + r, F - 1);            // rows past the last are not stored
  const int64_t esize = FP8 ? 1 : 2;
  const uint8_t* gate = p.gate_up + (expert * p.gu_stride + frow * p.gu_ld) * esize;
  const uint8_t* up = gate + F * p.gu_ld * esize;
  const uint16_t* xr[kTiles];
#pragma unroll
  for (int mt = 0; mt < kTiles; ++mt)
    xr[mt] = 16 * mt + r < n ? p.x + s_entry[16 * mt + r] / p.top_k * p.x_ld : nullptr;

  f32x4 ag[kTiles], au[kTiles];
#pragma unroll
  for (int mt = 0; mt < kTiles; ++mt) ag[mt] = au[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int lines = (K + W::kLine - 1) / W::kLine;
  const int per = (lines + kWaves - 1) / kWaves;
  const int first = wave * per, last = min(lines, first + per);
  constexpr int U = 4;                            // lines in flight
  for (int l = first; l < last; l += U) {
    uint4 wg[U][2], wu[U][2];
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int k = l + i < last ? (l + i) * W::kLine + (g + 4 * c) * W::kPer : K;
        wg[i][c] = W::load(gate, k, K);
        wu[i][c] = W::load(up, k, K);
      }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (l + i >= last) break;
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int v = 0; v < W::kMfma; ++v) {
          const int k = (l + i) * W::kLine + (g + 4 * c) * W::kPer + 8 * v;
          const bf16x8 fg = W::frag(wg[i][c], v), fu = W::frag(wu[i][c], v);
#pragma unroll
          for (int mt = 0; mt < kTiles; ++mt) {
            if (16 * mt >= n) break;
            bf16x8 fx = zero8();
            if (xr[mt] && k < K) fx = *reinterpret_cast<const bf16x8*>(xr[mt] + k);
            ag[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fg, fx, ag[mt], 0, 0, 0);
            au[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fu, fx, au[mt], 0, 0, 0);
          }
        }
    }
  }

  // Lane l holds rows 4 (l / 16) .. + 3 of the tile for the token of slot l % 16.
  const float scale = p.gate_up_scale ? p.gate_up_scale[expert] : 1.f;
  const ActCoef k = act_coef(p.act);
#pragma unroll
  for (int mt = 0; mt < kTiles; ++mt) {
    if (16 * mt >= n) break;
    if (mt) __syncthreads();
    *reinterpret_cast<f32x4*>(&s_red[0][wave][r][4 * g]) = ag[mt];
    *reinterpret_cast<f32x4*>(&s_red[1][wave][r][4 * g]) = au[mt];
    __syncthreads();
    const int slot = threadIdx.x >> 4, f = threadIdx.x & 15;
    if (threadIdx.x < 256 && 16 * mt + slot < n && f0 + f < F) {
      float zg = 0.f, zu = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        zg += s_red[0][w][slot][f];
        zu += s_red[1][w][slot][f];
      }
      float v = 0.f;
      with_act(p.act, [&](auto cls) { v = act_value<decltype(cls)::value>(k, zg * scale); });
      v *= zu * scale;
      const __bf16 hi = (__bf16)v;
      const float rest = __builtin_fabsf((float)hi) < __builtin_inff() ? v - (float)hi : 0.f;
      const __bf16 lo = (__bf16)rest;
      uint16_t* h = p.h + (int64_t)s_entry[16 * mt + slot] * F * 2 + (f0 + f) / 8 * 16 + (f0 + f) % 8;
      h[0] = __builtin_bit_cast(uint16_t, hi);
      h[8] = __builtin_bit_cast(uint16_t, lo);
    }
  }
#endif
}

// The down launch: one workgroup per 16 rows of the down weights (columns of y)
// and range of the (expert, K line) steps of the chosen experts; the steps of a
// range are cut over the waves.
template <bool FP8>
__global__ void __launch_bounds__(kThreads, 4) moe_down_kernel(MoeParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  using W = Weights<FP8>;
  constexpr int kSlots = kMoeMaxTokens * kMoeMaxTopK;
  __shared__ int32_t s_ids[kSlots];
  __shared__ float s_probs[kSlots];
  __shared__ int32_t s_used[kMoeMaxExperts];      // experts chosen at all, ascending
  __shared__ int32_t s_flag[kMoeMaxExperts];
  __shared__ int32_t s_count;
  __shared__ int32_t s_entry[kWaves][kMoeMaxTokens];
  __shared__ __attribute__((aligned(16))) float s_y[kWaves][kMoeMaxTokens][16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int slots = p.tokens * p.top_k;
  const int tile = blockIdx.x % p.tiles, split = blockIdx.x / p.tiles;
  for (int e = threadIdx.x; e < p.experts; e += kThreads) s_flag[e] = 0;
  for (int i = threadIdx.x; i < kWaves * p.tokens * 16; i += kThreads)
    s_y[i / (p.tokens * 16)][i / 16 % p.tokens][i & 15] = 0.f;
  __syncthreads();
  for (int i = threadIdx.x; i < slots; i += kThreads) {
    const int id = p.ws_ids[i];
    s_ids[i] = id;
    s_probs[i] = p.ws_probs[i];
    if (id >= 0) s_flag[id] = 1;
  }
  __syncthreads();
  if (wave == 0) {
    int n = 0;
    for (int e0 = 0; e0 < p.experts; e0 += 64) {
      const bool used = e0 + lane < p.experts && s_flag[e0 + lane];
      const uint64_t mask = __ballot(used);
      if (used) s_used[n + __builtin_popcountll(mask & ((1ull << lane) - 1))] = e0 + lane;
      n += __builtin_popcountll(mask);
    }
    if (lane == 0) s_count = n;
  }
  __syncthreads();

  const int K = p.ffn, D = p.hidden;
  const int d0 = 16 * tile, r = lane & 15, g = lane >> 4;
  const int drow = min(d0 + r, D - 1);
  const int64_t esize = FP8 ? 1 : 2;
  const int lines = (K + W::kLine - 1) / W::kLine;
  const int total = __builtin_amdgcn_readfirstlane(s_count) * lines;
  const int parts = p.splits * kWaves, part = split * kWaves + wave;
  int at = (int)((int64_t)total * part / parts);
  const int end = (int)((int64_t)total * (part + 1) / parts);
  while (at < end) {
    const int u = at / lines;
    const int l0 = at - u * lines, l1 = min(lines, l0 + end - at);
    at += l1 - l0;
    const int expert = __builtin_amdgcn_readfirstlane(s_used[u]);
    int n = 0;
    for (int c = 0; c < slots; c += 64) {
      const bool hit = c + lane < slots && s_ids[c + lane] == expert;
      const uint64_t mask = __ballot(hit);
      if (hit) s_entry[wave][n + __builtin_popcountll(mask & ((1ull << lane) - 1))] = c + lane;
      n += __builtin_popcountll(mask);
    }
    __builtin_amdgcn_wave_barrier();
    const uint8_t* row = p.down + (expert * p.down_stride + drow * p.down_ld) * esize;
    const uint16_t* hr[kTiles];
    f32x4 acc[kTiles];
#pragma unroll
    for (int mt = 0; mt < kTiles; ++mt) {
      hr[mt] = 16 * mt + r < n ? p.h + (int64_t)s_entry[wave][16 * mt + r] * K * 2 : nullptr;
      acc[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    constexpr int U = 4;
    for (int l = l0; l < l1; l += U) {
      uint4 w[U][2];
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c)
          w[i][c] = W::load(row, l + i < l1 ? (l + i) * W::kLine + (g + 4 * c) * W::kPer : K, K);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (l + i >= l1) break;
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int v = 0; v < W::kMfma; ++v) {
            const int k = (l + i) * W::kLine + (g + 4 * c) * W::kPer + 8 * v;
            const bf16x8 fw = W::frag(w[i][c], v);
#pragma unroll
            for (int mt = 0; mt < kTiles; ++mt) {
              if (16 * mt >= n) break;
              bf16x8 hi = zero8(), lo = zero8();
              if (hr[mt] && k < K) {
                hi = *reinterpret_cast<const bf16x8*>(hr[mt] + 2 * k);
                lo = *reinterpret_cast<const bf16x8*>(hr[mt] + 2 * k + 8);
              }
              acc[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw, hi, acc[mt], 0, 0, 0);
              acc[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw, lo, acc[mt], 0, 0, 0);
            }
          }
      }
    }
    const float scale = p.down_scale ? p.down_scale[expert] : 1.f;
#pragma unroll
    for (int mt = 0; mt < kTiles; ++mt) {
      if (16 * mt >= n) break;
      if (16 * mt + r < n) {
        const int i = s_entry[wave][16 * mt + r];
        const float w = s_probs[i] * scale;
        f32x4* y = reinterpret_cast<f32x4*>(&s_y[wave][i / p.top_k][4 * g]);
        *y += acc[mt] * w;
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  for (int i = threadIdx.x; i < p.tokens * 16; i += kThreads) {
    const int t = i >> 4, c = i & 15;
    if (d0 + c >= D) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += s_y[w][t][c];
    if (p.part) p.part[((int64_t)split * p.tokens + t) * D + d0 + c] = v;
    else p.y[t * p.y_ld + d0 + c] = __builtin_bit_cast(uint16_t, (__bf16)v);
  }
#endif
}

// The sum of the down product's ranges, in order.
__global__ void __launch_bounds__(256) moe_sum_kernel(MoeParams p) {
  const int64_t n = (int64_t)p.tokens * p.hidden;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  float v = 0.f;
  for (int s = 0; s < p.splits; ++s) v += p.part[s * n + i];
  const int64_t t = i / p.hidden;
  p.y[t * p.y_ld + (i - t * p.hidden)] = __builtin_bit_cast(uint16_t, (__bf16)v);
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
  p.splits = f.splits;
  const dim3 up((unsigned)f.up_workgroups), block(kThreads);
  if (s.fp8) hipLaunchKernelGGL(moe_up_kernel<true>, up, block, 0, stream, p);
  else hipLaunchKernelGGL(moe_up_kernel<false>, up, block, 0, stream, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  p.tiles = f.down_tiles;
  const dim3 down((unsigned)(f.down_tiles * f.splits));
  if (s.fp8) hipLaunchKernelGGL(moe_down_kernel<true>, down, block, 0, stream, p);
  else hipLaunchKernelGGL(moe_down_kernel<false>, down, block, 0, stream, p);
  e = hipGetLastError();
  if (e != hipSuccess || f.splits == 1) return e;
  hipLaunchKernelGGL(moe_sum_kernel, dim3((unsigned)((c.tokens * s.hidden + 255) / 256)), dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace ccl
