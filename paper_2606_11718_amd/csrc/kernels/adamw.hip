// AdamW over many tensors (ccl_adamw_step):
//   g <- grad * grad_scale;  m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2
//   p <- p (1 - lr wd) - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// in fp32, one pass over memory: 28 bytes an element with everything in fp32, 16
// with 8-bit moments and a bf16 gradient and copy. The tensors' table is a kernel
// argument, so that a step of small tensors is one launch and a captured step
// holds all it needs. Bound by memory: two tensors of 28672 x 8192 with 8-bit moments
// 1450 us (5.2 TB/s), their moments decoded 455 (6.2 TB/s), with fp32 ones 2526 (5.2), all
// in fp32 2481 (5.3), bf16 params and gradients with 8-bit moments 1108 (4.3); 60 tensors of 1.16 million
// elements together 9.7 us (3.4 TB/s), where the launch and the first loads count.
//
// 8-bit moments: 128 elements share a power of two, from the largest exponent
// among them. m is a sign, 4 exponent and 3 mantissa bits; v, never negative, 5
// and 3: m's smallest value is 2^-16 of the largest's power of two, v's 2^-32, whose
// root is 2^-16. Rounded up or down at random (a hash of the element's
// place and the step, so the same call gives the same bits): b2 = 0.999 moves v
// by a thousandth of itself a step, which rounding to the nearest of 3 mantissa
// bits would undo every time. Below its smallest value an m is then rounded up with
// the chance of its ratio to it, its v with that of the ratio's square, so that
// many live beside a v of 0: there v is taken as its smallest value when it is
// read, or m would be divided by eps alone (gradients of 1e-5 beside one of 1 in a
// block: steps of up to 700 learning rates, with that value 1.6, in fp32 1.0).
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "train_kernels.hpp"

namespace ccl {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// A tensor in the kernel's arguments, 4 KB of which hold kAdamwTensors.
struct Entry32 {
  void* param;
  const void* grad;
  void *m, *v;
  uint16_t* copy;
  int64_t n;
  float weight_decay;
  int32_t first;           // its first workgroup
};
struct Entry8 : Entry32 {
  uint8_t *m_scale, *v_scale;
};
template <bool BITS8>
struct AdamwTable {
  static constexpr int kTensors = kAdamwTensors[BITS8];
  std::conditional_t<BITS8, Entry8, Entry32> t[kTensors];
};
struct AdamwParams {
  const float *grad_scale, *lr_ptr;
  const int64_t* step_ptr;
  double lr, beta1, beta2;
  int64_t step;
  float b1, c1, b2, c2, eps;       // c: 1 - b
  float rate, root;                // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  int32_t count, chunk;            // elements of a workgroup
};

// The same 32 bits for the same element and step.
__device__ __forceinline__ uint32_t chance(int64_t i, uint32_t seed) {
  uint32_t h = (uint32_t)i + ((uint32_t)(i >> 32) << 7);
  h = h * 0x9E3779B1u + seed;
  h ^= h >> 16;
  h *= 0x6A09E667u;
  h ^= h >> 13;
  h *= 0xBB67AE85u;
  return h ^ (h >> 16);
}

__device__ __forceinline__ float power2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Moment formats: exponent bits E, 3 mantissa bits. A block's values are brought
// below 2^(kReach + 1); kBias is the format's.
template <int E>
struct Moment {
  static constexpr int kReach = E == 4 ? 7 : 14, kBias = E == 4 ? 7 : 16;
  static constexpr uint32_t kNan = E == 4 ? 0x7f : 0xff;
  // Code bits as the top bits of an fp32 with exponent bias 127, brought to kBias:
  // the format's subnormal values are fp32's.
  __device__ static __forceinline__ float decode(uint32_t code, int top) {
    const uint32_t c = E == 4 ? code & 127 : code;
    float y = __uint_as_float(c << 20) * power2(127 - kBias);
    if (c == kNan) y = __uint_as_float(0x7fc00000u);
    if (E == 4 && code & 128) y = -y;
    return y * power2(top - 127 - kReach);
  }
  __device__ static __forceinline__ int scale(int top) { return max(top, kReach + 1); }
  __device__ static __forceinline__ uint32_t encode(float x, int top, uint32_t random16) {
    constexpr int kLow = 1 - kBias;
    const uint32_t bits = __float_as_uint(x);
    const float y = __uint_as_float(bits & 0x7fffffffu) * power2(kReach + 127 - top);
    const int e = max((int)(__float_as_uint(y) >> 23) - 127, kLow);
    const float steps = y * power2(3 - e) + (float)random16 * (1.f / 65536.f);
    uint32_t code = (uint32_t)(int)steps + (uint32_t)((e - kLow) << 3);
    if ((bits & 0x7f800000u) == 0x7f800000u) code = kNan;      // infinite or NaN
    if (E == 4 && x < 0.f) code |= 128;
    return code;
  }
};
// The biased exponent of |x|, 0 where it is not finite.
__device__ __forceinline__ int exponent_of(float x) {
  const int e = (__float_as_uint(x) >> 23) & 255;
  return e == 255 ? 0 : e;
}

// Eight consecutive elements as fp32 and back; n of them exist.
template <bool BF16>
__device__ __forceinline__ void load8(const void* base, int64_t at, int n, bool whole, float (&v)[8]) {
  if constexpr (BF16) {
    const uint16_t* p = static_cast<const uint16_t*>(base) + at;
    if (whole) {
      const uint4 a = *reinterpret_cast<const uint4*>(p);
      const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(w[j] << 16);
        v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = j < n ? __uint_as_float((uint32_t)p[j] << 16) : 0.f;
    }
  } else {
    const float* p = static_cast<const float*>(base) + at;
    if (whole) {
      const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = a[j];
        v[4 + j] = b[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = j < n ? p[j] : 0.f;
    }
  }
}

__device__ __forceinline__ uint4 to_bf16x8(const float (&v)[8]) {
  typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
  typedef float f32x8 __attribute__((ext_vector_type(8)));
  f32x8 x;
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = v[j];
  return __builtin_bit_cast(uint4, __builtin_convertvector(x, bf16x8));     // nearest even, NaN kept
}

template <bool BF16>
__device__ __forceinline__ void store8(void* base, int64_t at, int n, bool whole, const float (&v)[8]) {
  if constexpr (BF16) {
    uint16_t* p = static_cast<uint16_t*>(base) + at;
    const uint4 b = to_bf16x8(v);
    if (whole) {
      *reinterpret_cast<uint4*>(p) = b;
    } else {
      const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) p[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
    }
  } else {
    float* p = static_cast<float*>(base) + at;
    if (whole) {
      reinterpret_cast<f32x4*>(p)[0] = f32x4{v[0], v[1], v[2], v[3]};
      reinterpret_cast<f32x4*>(p)[1] = f32x4{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) p[j] = v[j];
    }
  }
}

__device__ __forceinline__ uint2 load_codes(const uint8_t* p, int n, bool whole) {
  if (whole) return *reinterpret_cast<const uint2*>(p);
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < n) w[j >> 2] |= (uint32_t)p[j] << (8 * (j & 3));
  return make_uint2(w[0], w[1]);
}

__device__ __forceinline__ void store_codes(uint8_t* p, int n, bool whole, uint2 c) {
  if (whole) {
    *reinterpret_cast<uint2*>(p) = c;
    return;
  }
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < n) p[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
}

__device__ __forceinline__ uint32_t code_of(uint2 c, int j) { return ((j < 4 ? c.x : c.y) >> (8 * (j & 3))) & 255; }

// v's codes with 1, the smallest value, in place of 0 where m's code is not a 0.
__device__ __forceinline__ uint32_t taken_v(uint32_t v, uint32_t m) {
  const uint32_t live = (m & 0x7f7f7f7fu) + 0x7f7f7f7fu, some = ((v & 0x7f7f7f7fu) + 0x7f7f7f7fu) | v;
  return v | ((live & ~some & 0x80808080u) >> 7);
}
__device__ __forceinline__ uint2 taken_v(uint2 v, uint2 m) { return make_uint2(taken_v(v.x, m.x), taken_v(v.y, m.y)); }

// The largest of a block's 16 threads.
__device__ __forceinline__ int block_top(const float (&x)[8]) {
  int top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, exponent_of(x[j]));
#pragma unroll
  for (int s = 1; s < 16; s <<= 1) top = max(top, __shfl_xor(top, s));
  return top;
}

template <int E>
__device__ __forceinline__ void decode8(uint2 codes, int top, float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = Moment<E>::decode(code_of(codes, j), top);
}

template <int E>
__device__ __forceinline__ uint2 encode8(const float (&x)[8], int top, const uint32_t (&random)[8], int shift) {
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j >> 2] |= Moment<E>::encode(x[j], top, (random[j] >> shift) & 0xffff) << (8 * (j & 3));
  return make_uint2(w[0], w[1]);
}

__device__ __forceinline__ bool aligned_to(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// TINY: subnormal numbers have a root. v_sqrt_f32 takes them as 0; their roots, below
// 2^-63, are nothing beside an eps of 1e-8, but without an eps m would be divided by 0.
// (A kernel of its own: 28672 x 8192 twice with 8-bit moments takes 1928 us so, 1890
// without, and 1906 with a uniform branch in one kernel.)
template <bool P16, bool G16, bool BITS8, bool TINY>
__global__ void __launch_bounds__(256) adamw_kernel(AdamwTable<BITS8> table, AdamwParams a) {
// Products and sums round one by one, as their formulas say: the 8-bit codes are
// the same wherever they are computed.
#pragma clang fp contract(off)
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (table.t[mid].first <= (int32_t)blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  const auto& t = table.t[lo];
  const int64_t n = t.n, from = (int64_t)((int32_t)blockIdx.x - t.first) * a.chunk;
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  if (!(__builtin_fabsf(gs) < INFINITY)) return;      // a step to be left out
  double lr = a.lr;
  float rate = a.rate, root = a.root;
  int64_t step = a.step;
  if (a.lr_ptr || a.step_ptr) {
    if (a.lr_ptr) lr = *a.lr_ptr;
    if (a.step_ptr) step = *a.step_ptr;
    if (!(__builtin_fabs(lr) < (double)INFINITY) || step < 1) return;
    rate = (float)(lr / (1.0 - power_of(a.beta1, step)));
    root = (float)(1.0 / sqrt(1.0 - power_of(a.beta2, step)));
  }
  const float keep = (float)(1.0 - lr * (double)t.weight_decay);
  const uint32_t seed = (uint32_t)step * 0x3C6EF373u;
  const bool fit = aligned_to(t.param, 16) && aligned_to(t.grad, 16) && aligned_to(t.m, BITS8 ? 8 : 16) &&
                   aligned_to(t.v, BITS8 ? 8 : 16) && aligned_to(t.copy, 16);
  const int64_t end = from + a.chunk < n ? from + a.chunk : n;
  for (int64_t at = from + threadIdx.x * 8; at - threadIdx.x % 16 * 8 < end; at += 256 * 8) {
    const int left = (int)(end - at < 8 ? end - at : 8);     // may be none in a block's last threads
    const bool whole = fit && left == 8;
    float p[8], g[8], m[8], v[8];
    load8<P16>(t.param, at, left, whole, p);
    load8<G16>(t.grad, at, left, whole, g);
    if constexpr (BITS8) {
      const int64_t block = at / kAdamwBlock;
      const uint2 mc = load_codes(static_cast<const uint8_t*>(t.m) + at, left, whole);
      const uint2 vc = load_codes(static_cast<const uint8_t*>(t.v) + at, left, whole);
      decode8<4>(mc, Moment<4>::scale(t.m_scale[block]), m);
      decode8<5>(taken_v(vc, mc), Moment<5>::scale(t.v_scale[block]), v);
    } else {
      load8<false>(t.m, at, left, whole, m);
      load8<false>(t.v, at, left, whole, v);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = g[j] * gs;
      m[j] = m[j] * a.b1 + x * a.c1;
      v[j] = v[j] * a.b2 + (x * x) * a.c2;
      // v_sqrt_f32 and v_rcp_f32, 1 ulp each: far below the rounding of p
      float r = __builtin_amdgcn_sqrtf(v[j]);
      if (TINY && v[j] < 0x1p-126f) r = __builtin_amdgcn_sqrtf(v[j] * 0x1p64f) * 0x1p-32f;
      const float d = r * root + a.eps;
      p[j] = p[j] * keep - m[j] * rate * __builtin_amdgcn_rcpf(d);
    }
    store8<P16>(t.param, at, left, whole, p);
    if (t.copy) store8<true>(t.copy, at, left, whole, p);
    if constexpr (BITS8) {
      uint32_t random[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) random[j] = chance(at + j, seed);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j >= left) m[j] = v[j] = 0.f;
      const int mt = Moment<4>::scale(block_top(m)), vt = Moment<5>::scale(block_top(v));
      store_codes(static_cast<uint8_t*>(t.m) + at, left, whole, encode8<4>(m, mt, random, 0));
      store_codes(static_cast<uint8_t*>(t.v) + at, left, whole, encode8<5>(v, vt, random, 16));
      if (threadIdx.x % 16 == 0) {
        t.m_scale[at / kAdamwBlock] = (uint8_t)mt;
        t.v_scale[at / kAdamwBlock] = (uint8_t)vt;
      }
    } else {
      store8<false>(t.m, at, left, whole, m);
      store8<false>(t.v, at, left, whole, v);
    }
  }
}

template <bool BF16>
__global__ void __launch_bounds__(256) moments_kernel(int64_t n, const uint8_t* m, const uint8_t* m_scale, const uint8_t* v,
                                                      const uint8_t* v_scale, void* m_out, void* v_out) {
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (at >= n) return;
  const int left = (int)(n - at < 8 ? n - at : 8);
  float x[8];
  const uint2 mc = m ? load_codes(m + at, left, left == 8 && aligned_to(m, 8)) : make_uint2(0, 0);
  if (m_out) {
    decode8<4>(mc, Moment<4>::scale(m_scale[at / kAdamwBlock]), x);
    store8<BF16>(m_out, at, left, left == 8 && aligned_to(m_out, 16), x);
  }
  if (v_out) {
    const uint2 vc = load_codes(v + at, left, left == 8 && aligned_to(v, 8));
    decode8<5>(taken_v(vc, mc), Moment<5>::scale(v_scale[at / kAdamwBlock]), x);
    store8<BF16>(v_out, at, left, left == 8 && aligned_to(v_out, 16), x);
  }
}

}  // namespace

namespace {

template <bool P16, bool G16, bool BITS8, bool TINY>
hipError_t launch(AdamwParams a, const AdamwTensor* tensors, int64_t count, hipStream_t stream) {
  using Table = AdamwTable<BITS8>;
  static_assert(sizeof(Table) + sizeof(AdamwParams) <= 4096, "kernel arguments");
  for (int64_t i = 0; i < count;) {
    Table table;
    int64_t groups = 0, elems = 0;
    int k = 0;
    // 8192 elements of a workgroup; 2048, one pass, while that is few workgroups
    for (int64_t j = i; j < count && j < i + Table::kTensors; ++j) elems += tensors[j].n;
    a.chunk = elems <= 2048 * 4096 ? 2048 : 8192;
    for (; i < count && k < Table::kTensors; ++i) {
      const AdamwTensor& s = tensors[i];
      const int64_t need = (s.n + a.chunk - 1) / a.chunk;
      if (k && groups + need > 0xffffff) break;       // fewer than 2^32 threads
      auto& t = table.t[k++];
      t.param = s.param;
      t.grad = s.grad;
      t.m = s.m;
      t.v = s.v;
      t.copy = s.copy;
      t.n = s.n;
      t.weight_decay = s.weight_decay;
      t.first = (int32_t)groups;
      if constexpr (BITS8) {
        t.m_scale = s.m_scale;
        t.v_scale = s.v_scale;
      }
      groups += need;
    }
    a.count = k;
    hipLaunchKernelGGL((adamw_kernel<P16, G16, BITS8, TINY>), dim3((unsigned)groups), dim3(256), 0, stream, table, a);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_adamw(const AdamwStep& s, const AdamwTensor* tensors, int64_t count, bool p_bf16, bool g_bf16, bool bits8,
                        hipStream_t stream) {
  AdamwParams a{};
  a.grad_scale = s.grad_scale;
  a.lr_ptr = s.lr_ptr;
  a.step_ptr = s.step_ptr;
  a.lr = s.lr;
  a.beta1 = s.beta1;
  a.beta2 = s.beta2;
  a.step = s.step;
  a.b1 = (float)s.beta1;
  a.c1 = (float)(1.0 - s.beta1);
  a.b2 = (float)s.beta2;
  a.c2 = (float)(1.0 - s.beta2);
  a.eps = (float)s.eps;
  if (!s.step_ptr) {
    a.rate = (float)(s.lr / (1.0 - power_of(s.beta1, s.step)));
    a.root = (float)(1.0 / sqrt(1.0 - power_of(s.beta2, s.step)));
  }
  // a subnormal's root, below 2^-63, over sqrt(1 - b2^t) is less than 2^-24 of eps
  const bool tiny = !(s.eps * sqrt(1.0 - s.beta2) >= 0x1p-39);
  const auto kind = [&](auto p16, auto g16) {
    constexpr bool P = decltype(p16)::value, G = decltype(g16)::value;
    if (tiny) return bits8 ? launch<P, G, true, true>(a, tensors, count, stream) : launch<P, G, false, true>(a, tensors, count, stream);
    return bits8 ? launch<P, G, true, false>(a, tensors, count, stream) : launch<P, G, false, false>(a, tensors, count, stream);
  };
  const std::true_type yes;
  const std::false_type no;
  return p_bf16 ? (g_bf16 ? kind(yes, yes) : kind(yes, no)) : (g_bf16 ? kind(no, yes) : kind(no, no));
}

hipError_t launch_adamw_moments(int64_t n, const uint8_t* m, const uint8_t* m_scale, const uint8_t* v, const uint8_t* v_scale,
                                void* m_out, void* v_out, bool bf16, hipStream_t stream) {
  const dim3 grid((unsigned)((n + 2047) / 2048));
  if (bf16) hipLaunchKernelGGL(moments_kernel<true>, grid, dim3(256), 0, stream, n, m, m_scale, v, v_scale, m_out, v_out);
  else hipLaunchKernelGGL(moments_kernel<false>, grid, dim3(256), 0, stream, n, m, m_scale, v, v_scale, m_out, v_out);
  return hipGetLastError();
}

}  // namespace ccl
