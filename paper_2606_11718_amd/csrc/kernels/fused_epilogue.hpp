// Epilogues of ccl_gemm_fused and ccl_gemm_fused_grad on a tile of the
// product D = A B. Included by gemm.hip inside its namespace.
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
};

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

// The simple form: the product's fp32 partial tiles (split-K ranges, or one
// range of the whole K) are read back from the workspace and summed in
// ascending range order, one float4 per thread, as splitk_reduce_kernel does.
// Bound by reading the partials; used for split-K and for the plans whose
// GEMM kernel has no fused epilogue of its own.
template <int BM, int BN, int WGN, int MD, int WGM, bool GRAD>
__global__ void __launch_bounds__(256) fused_reduce_kernel(FusedParams p) {
  using L = AccLayout<MD>;
  constexpr int WM = BM / WGM, WN = BN / WGN;
  constexpr int TM = WM / MD, TN = WN / MD;
  constexpr int kChunks = BM * BN / (4 * 256);
  const int64_t slot = blockIdx.x >> 3;
  const int32_t chunk = (int32_t)(slot % kChunks);
  int32_t pr, pc, ti, tj, split;
  if (!map_tile(p.map, ((slot / kChunks) << 3) | (blockIdx.x & 7), &pr, &pc, &ti, &tj, &split)) return;
  const int32_t f = chunk * 256 + threadIdx.x;
  const int lane = f & 63;
  int r = f >> 6;
  const int q = r % L::Q;
  r /= L::Q;
  const int nt = r % TN;
  r /= TN;
  const int mt = r % TM;
  const int wave = r / TM;
  const int wm = wave / (BN / WN), wn = wave % (BN / WN);
  const int64_t m = ti * BM + wm * WM + mt * MD + L::row(lane);   // row in the partition
  const int n = tj * BN + wn * WN + nt * MD + L::col(lane, q);    // column of D in the partition
  const FusedEpi& e = p.e;
  const bool live = pr * e.part_rows + m < e.rows;
  const int32_t S = p.splits_total;
  const float4* part = reinterpret_cast<const float4*>(p.ws + tile_id(p, pr, pc, ti, tj) * S * (BM * BN));
  auto sum = [&](int32_t at) {
    f32x4 o{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < S; ++s) o += *reinterpret_cast<const f32x4*>(part + at + (int64_t)s * (BM * BN / 4));
    return o * p.alpha;
  };
  const int64_t c_at = pr * p.c.part + pc * p.c.slice + m * p.c.ld;
  const int64_t z_at = pr * e.z.part + pc * e.z.slice + m * e.z.ld;
  auto put = [](uint16_t* base, int64_t at, f32x4 v) { *reinterpret_cast<uint2*>(base + at) = f32_to_bf16x4(v); };
  uint16_t* C = static_cast<uint16_t*>(p.C);
  const f32x4 zero{0.f, 0.f, 0.f, 0.f};
  if constexpr (!GRAD) {
    // The up columns' threads leave: the gate columns' threads read both. The
    // up's float4 lies in the next MFMA tile (16 wide) or two groups on (32).
    constexpr int kUp = MD == 16 ? 64 * L::Q : 2 * 64;
    if (e.gated && (n & 16)) return;
    f32x4 z = live ? sum(f) + bias4(e, pc * (int64_t)e.part_cols + n) : zero;
    f32x4 u = e.gated && live ? sum(f + kUp) + bias4(e, pc * (int64_t)e.part_cols + n + 16) : zero;
    if (e.Zout) {
      put(e.Zout, z_at + n, z);
      if (e.gated) put(e.Zout, z_at + n + 16, u);
    }
    f32x4 o;
    with_act(e.act, [&](auto act) {
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = act_value<decltype(act)::value>(z[j]);
    });
    if (e.gated) o *= u;
    const int cn = e.gated ? ((n >> 5) << 4) | (n & 15) : n;
    if (!live) {
      o = zero;
    } else if (e.R) {
      const f32x4 res = bf16x4_to_f32(*reinterpret_cast<const uint2*>(e.R + c_at + cn));
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = __builtin_fmaf(e.beta, res[j], o[j]);
    }
    put(C, c_at + cn, o);
  } else {
    const int zn = e.gated ? wide_col(n) : n;
    f32x4 g = zero, u = zero;
    if (live) {
      const f32x4 d = sum(f);
      const f32x4 z = e.Zin ? bf16x4_to_f32(*reinterpret_cast<const uint2*>(e.Zin + z_at + zn)) : zero;
      const f32x4 zu = e.gated ? bf16x4_to_f32(*reinterpret_cast<const uint2*>(e.Zin + z_at + zn + 16)) : zero;
      with_act(e.act, [&](auto act) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float grad;
          const float value = act_value_grad<decltype(act)::value>(z[j], &grad);
          g[j] = d[j] * grad;
          if (e.gated) {
            g[j] *= zu[j];
            u[j] = d[j] * value;
          }
        }
      });
    }
    put(C, c_at + zn, g);
    if (e.gated) put(C, c_at + zn + 16, u);
    if (e.colsum) {
      // The MD lanes of a column group hold MD rows of four columns.
      const int64_t block = (pr * e.part_rows + m) / MD;
      float* to = e.colsum + block * e.z_cols + (e.gated ? 2 : 1) * pc * (int64_t)e.part_cols + zn;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (half && !e.gated) break;
        f32x4 v = half ? u : g;
#pragma unroll
        for (int x = 1; x < MD; x <<= 1)
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] += __shfl_xor(v[j], x);
        if ((lane & (MD - 1)) == 0) *reinterpret_cast<f32x4*>(to + 16 * half) = v;
      }
    }
  }
}

// Column sums over the row blocks, in a fixed order: thread (g, c) adds the
// blocks g, g + 4, ... of its column, then the four are added.
__global__ void __launch_bounds__(256) bias_reduce_kernel(const float* part, int64_t blocks, int64_t cols, float* out) {
  __shared__ float sm[4][64];
  const int c = threadIdx.x & 63, g = threadIdx.x >> 6;
  const int64_t col = (int64_t)blockIdx.x * 64 + c;
  float v = 0.f;
  if (col < cols) {
#pragma unroll 8
    for (int64_t b = g; b < blocks; b += 4) v += part[b * cols + col];
  }
  sm[g][c] = v;
  __syncthreads();
  if (g == 0 && col < cols) out[col] = ((sm[0][c] + sm[1][c]) + sm[2][c]) + sm[3][c];
}
