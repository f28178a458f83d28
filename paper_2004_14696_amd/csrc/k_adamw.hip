// AdamW over many tensors: one step is
//   k_adamw_norm   (only where a norm is asked for) sums of squares of g,
//   k_adamw_prep   one workgroup: t, the norm, the clip factor, 1 - beta^t,
//   k_adamw_update every tensor, a workgroup to a chunk of 1024 values.
//
// The update moves 8 bytes of w, 16 (32-bit states) or 4 + 1/64 (8-bit) of
// states, and the gradient, each once, and is bound by that: 5.5 TB/s with
// either.  With 8-bit states only just: 133 vector instructions a value took
// 425 us for 128M values, 77 take 374 (codes by the stochastic conversion, a
// shorter root, one product of the hash for four values, no 64-bit division).
// In calls right behind each other their power lowers the clock: the step of
// 450 us takes 550 after ten, and 470 in the long run (690 and 525 before);
// 32-bit states keep their time.
//
// A lane holds four consecutive values (16 bytes of w), a wave the 256 values of
// one scale, so the largest magnitude of a block is a reduction over the lanes
// of one wave and nothing goes through shared memory.  The table of chunks gives
// a workgroup its tensor with one load, whatever the sizes of the tensors.
// 64M values, 32-bit states, fp16 gradients and copy: 329 us, 5.5 TB/s (chunks of
// 4096 values 357: fewer loads under way); 128M, 8-bit states, bf16 gradients
// and copy, clipped: 447 us, 374 of them the update and 66 the norm (3.9 TB/s);
// 0.4M values, clipped: 14 us, three launches.
//
// t and what depends on it live on the device (a captured step advances them
// at every replay) and are handed from kernel to kernel in stream order: no
// atomics, no waits between workgroups, sums in a fixed order.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "lm_ops.h"

namespace dbw {
namespace {

constexpr int kThreads = 256;
constexpr int kNormChunks = 4;   // chunks that a workgroup of the norm has in flight

template <typename G>
struct Vec4;   // four gradients
template <>
struct Vec4<float> {
  static __device__ __forceinline__ void load(const float* p, float (&x)[4]) {
    const lm_f32x4 v = *reinterpret_cast<const lm_f32x4_any*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = v[j];
  }
};
template <typename H>
struct Vec4Half {
  typedef H V __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ void load(const H* p, float (&x)[4]) {
    const V v = __builtin_bit_cast(V, static_cast<lm_u32x2>(*reinterpret_cast<const lm_u32x2_any*>(p)));
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = static_cast<float>(v[j]);
  }
};
template <>
struct Vec4<__bf16> : Vec4Half<__bf16> {};
template <>
struct Vec4<_Float16> : Vec4Half<_Float16> {};

// `n` (at most 4) values at p; the others 0.
template <typename G>
__device__ __forceinline__ void load4(const G* p, int n, float (&x)[4]) {
  if (n >= 4) {
    Vec4<G>::load(p, x);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = j < n ? lm_to_f32(p[j]) : 0.f;
  }
}
__device__ __forceinline__ void store4(float* p, int n, const float (&x)[4]) {
  if (n >= 4) {
    *reinterpret_cast<lm_f32x4_any*>(p) = lm_f32x4{x[0], x[1], x[2], x[3]};
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[j] = x[j];
  }
}
template <typename H>
__device__ __forceinline__ void store4_half(H* p, int n, const float (&x)[4]) {
  typedef H V __attribute__((ext_vector_type(4)));
  if (n >= 4) {
    const V v = __builtin_convertvector(lm_f32x4{x[0], x[1], x[2], x[3]}, V);
    *reinterpret_cast<lm_u32x2_any*>(p) = __builtin_bit_cast(lm_u32x2, v);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[j] = static_cast<H>(x[j]);
  }
}

typedef uint32_t u32_any __attribute__((aligned(1)));
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int n) {
  if (n >= 4) return *reinterpret_cast<const u32_any*>(p);
  uint32_t v = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j < n) v |= static_cast<uint32_t>(p[j]) << (8 * j);
  return v;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int n, uint32_t v) {
  if (n >= 4) {
    *reinterpret_cast<u32_any*>(p) = v;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[j] = static_cast<uint8_t>(v >> (8 * j));
  }
}

__device__ __forceinline__ float pow2(int e) { return __builtin_bit_cast(float, static_cast<uint32_t>(e + 127) << 23); }

// Four e4m3 codes times 2^(e - 127).
__device__ __forceinline__ void decode(uint32_t codes, uint32_t e, float (&x)[4]) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false);
  const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
  const float s = e ? pow2(static_cast<int>(e) - 127) : 0x1p-127f;
  x[0] = a[0] * s;
  x[1] = a[1] * s;
  x[2] = b[0] * s;
  x[3] = b[1] * s;
}

// The largest of the 64 lanes' v, in all of them (a scalar).
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  const auto with = [&](auto ctrl, auto rows) {
    const uint32_t o = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(
        0, static_cast<int>(v), decltype(ctrl)::value, decltype(rows)::value, 0xf, true));
    v = v > o ? v : o;
  };
  typedef std::integral_constant<int, 0xf> all;
  with(std::integral_constant<int, 0x111>{}, all{});   // the lanes 1, 2, 4 and 8 before, in rows of 16
  with(std::integral_constant<int, 0x112>{}, all{});
  with(std::integral_constant<int, 0x114>{}, all{});
  with(std::integral_constant<int, 0x118>{}, all{});
  with(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // a row's last lane, to the next row
  with(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});   // the first half's, to the second
  return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), 63));
}

constexpr uint32_t kInf = 0x7f800000u;
__device__ __forceinline__ uint32_t abs_bits(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }
// Magnitudes as integers: their order is that of the values, with infinities
// and NaN on top.  The least leaves out zeros (which wrap around).
__device__ __forceinline__ uint32_t lane_most(const float (&x)[4]) {
  const uint32_t a = max(abs_bits(x[0]), abs_bits(x[1])), b = max(abs_bits(x[2]), abs_bits(x[3]));
  return max(a, b);
}
__device__ __forceinline__ uint32_t lane_least(const float (&x)[4]) {
  const uint32_t a = min(abs_bits(x[0]) - 1u, abs_bits(x[1]) - 1u), b = min(abs_bits(x[2]) - 1u, abs_bits(x[3]) - 1u);
  return min(a, b);
}

// Codes of the 256 values of a wave, four a lane, and the biased exponent of
// their scale.  `most`: wave_max of lane_most(x).  `bits`: a value's 16
// random bits, above 16 zeros (the conversion would look at four of those).
// FLOOR: what is above 0 stays above 0.
//
// Where all values are finite and none but zeros is below 2^-6 in units of the
// scale, the conversion with stochastic rounding gives the formula's codes, sign
// included (a test compares all floats of [2^-6, 448], each with bits of the
// mix; of smaller values some pairs differ, where the formula's sum in fp32 is
// rounded).  It takes one instruction a value for some fifteen.
template <bool FLOOR>
__device__ __forceinline__ uint32_t encode(const float (&x)[4], const uint32_t (&bits)[4], uint32_t most,
                                           uint32_t* scale) {
  const bool finite = most < kInf;
  if (!finite) {
    uint32_t lane = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) lane = max(lane, abs_bits(x[j]) < kInf ? abs_bits(x[j]) : 0u);
    most = wave_max(lane);
  }
  const uint32_t tb = max(most, __builtin_bit_cast(uint32_t, 0x1p-118f));
  // the largest value times 2^-e is in (224, 448]: 448 = 1.75 2^8 is the
  // largest code
  const int e = static_cast<int>(tb >> 23) - 127 - 8 + ((tb & 0x7fffffu) > 0x600000u ? 1 : 0);
  *scale = static_cast<uint32_t>(e + 127);
  const float inv = pow2(-e);
  uint32_t codes = 0;
  // 2^(e - 6): 0 or a subnormal's bits are below those of any normal value
  const uint32_t low = e - 6 > -127 ? static_cast<uint32_t>(e - 6 + 127) << 23 : 1u << 23;
  if (finite && __all(lane_least(x) >= low - 1u)) {
    codes = __builtin_amdgcn_cvt_sr_fp8_f32(x[0] * inv, bits[0], codes, 0);
    codes = __builtin_amdgcn_cvt_sr_fp8_f32(x[1] * inv, bits[1], codes, 1);
    codes = __builtin_amdgcn_cvt_sr_fp8_f32(x[2] * inv, bits[2], codes, 2);
    codes = __builtin_amdgcn_cvt_sr_fp8_f32(x[3] * inv, bits[3], codes, 3);
    return codes;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float y = fabsf(x[j]) * inv;                       // exact, or below every code
    // 2^(step) is the distance of the codes at y: 8 to a power of two, down
    // to 2^-6, evenly spaced below
    const int ey = static_cast<int>(__builtin_bit_cast(uint32_t, fmaxf(y, 0x1p-6f)) >> 23) - 127;
    uint32_t q = static_cast<uint32_t>(y * pow2(3 - ey) + static_cast<float>(bits[j] >> 16) * 0x1p-16f);
    if (FLOOR) q = q == 0 && x[j] > 0.f ? 1u : q;
    uint32_t c = static_cast<uint32_t>((ey + 6) * 8) + q;    // a carry of q moves to the next power
    c = fabsf(x[j]) <= 0x1.fffffep127f ? c : 0x7fu;
    c |= __builtin_bit_cast(uint32_t, x[j]) >> 24 & 0x80u;
    codes |= c << (8 * j);
  }
  return codes;
}

// sqrt(v), correctly rounded for v = 0 and from 2^-100 to 2^127: y is within an
// ulp or so of 1/sqrt(v), g of sqrt(v), and one Newton step with its residual,
// which is exact in a fused multiply-add, gives the rounded root (Markstein,
// "Computation of elementary functions on the IBM RISC System/6000", 1990; a
// test compares updates by 2^24 roots at five powers of four with those by
// sqrtf).  Other v that are not 0 give a root
// below 2^-50, an infinity or a NaN.
__device__ __forceinline__ float root(float v) {
  const float y = __builtin_amdgcn_rsqf(fmaxf(v, 0x1p-100f));
  const float g = v * y;
  return fmaf(fmaf(-g, g, v), 0.5f * y, g);
}

template <typename G>
__global__ __launch_bounds__(kThreads) void k_adamw_norm(const AdamTensor* __restrict__ tensors,
                                                         const AdamChunk* __restrict__ chunks, int64_t nchunks,
                                                         double* __restrict__ parts) {
  // squares and their sums in 64 bits: products of two fp32 values are exact
  // there, and neither overflow nor a long sum loses the small tensors
  double sum = 0.0;
  for (int64_t c = static_cast<int64_t>(blockIdx.x) * kNormChunks; c < nchunks;
       c += static_cast<int64_t>(gridDim.x) * kNormChunks) {
    float x[kNormChunks][4];
#pragma unroll
    for (int q = 0; q < kNormChunks; ++q) {
      // (behind the last chunk: that one again, with nothing left of it)
      const AdamChunk ch = chunks[c + q < nchunks ? c + q : nchunks - 1];
      const int64_t at = static_cast<int64_t>(ch.index) * kAdamChunk + threadIdx.x * 4;
      const int64_t left = c + q < nchunks ? tensors[ch.tensor].count - at : 0;
      load4(static_cast<const G*>(tensors[ch.tensor].g) + at, static_cast<int>(left < 4 ? left : 4), x[q]);
    }
#pragma unroll
    for (int q = 0; q < kNormChunks; ++q)
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += static_cast<double>(x[q][j]) * static_cast<double>(x[q][j]);
  }
#pragma unroll
  for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
  __shared__ double waves[kThreads / 64];
  if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x == 0) parts[blockIdx.x] = (waves[0] + waves[1]) + (waves[2] + waves[3]);
}

__global__ __launch_bounds__(kThreads) void k_adamw_prep(AdamStep* step, const double* __restrict__ parts, int nparts,
                                                         dbw_adamw_hyper h, float* norm_out) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < nparts; i += kThreads) sum += parts[i];
#pragma unroll
  for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
  __shared__ double waves[kThreads / 64];
  if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x != 0) return;
  const double norm = fabs(h.grad_scale) * sqrt((waves[0] + waves[1]) + (waves[2] + waves[3]));
  double f = h.grad_scale;
  int skip = 0;
  if (nparts && h.max_norm > 0.0) {
    skip = !(norm <= 0x1.fffffffffffffp1023);
    if (norm > h.max_norm) f *= h.max_norm / norm;
  }
  if (norm_out) *norm_out = static_cast<float>(norm);
  const int64_t t = step->t + (skip ? 0 : 1);
  step->t = t;
  step->skip = skip;
  // a factor near fp32's smallest values would lose its digits there: it goes in
  // two, the first of which loses none of a gradient that matters
  const double pre = fabs(f) < 0x1p-100 ? 0x1p-64 : 1.0;
  step->f = static_cast<float>(f / pre);
  step->pre = static_cast<float>(pre);
  step->ibc1 = 1.0 / (1.0 - pow(h.beta1, static_cast<double>(t)));
  step->ibc2 = static_cast<float>(1.0 / sqrt(1.0 - pow(h.beta2, static_cast<double>(t))));
  step->key = adam_mix(adam_mix(h.seed) + static_cast<uint32_t>(t));
}

template <typename G, int BITS>
__global__ __launch_bounds__(kThreads) void k_adamw_update(const AdamTensor* __restrict__ tensors,
                                                           const AdamChunk* __restrict__ chunks,
                                                           const AdamStep* __restrict__ step, dbw_adamw_hyper h,
                                                           int low_dtype) {
  // m and v in the order of their formulas, every product and sum rounded by
  // itself: the stored codes are then those of the formula in fp32
#pragma clang fp contract(off)
  if (step->skip) return;
  const AdamChunk ch = chunks[blockIdx.x];
  const AdamTensor t = tensors[ch.tensor];
  const int64_t first = static_cast<int64_t>(ch.index) * kAdamChunk;
  const int64_t left = t.count - first;
  const double lr = h.lr * t.lr_scale;
  const float f = step->f, pre = step->pre, ibc2 = step->ibc2, eps = static_cast<float>(h.eps);
  const float keep = static_cast<float>(1.0 - lr * t.decay), rate = static_cast<float>(lr * step->ibc1);
  const float b1 = static_cast<float>(h.beta1), c1 = static_cast<float>(1.0 - h.beta1);
  const float b2 = static_cast<float>(h.beta2), c2 = static_cast<float>(1.0 - h.beta2);
  const uint32_t key = BITS == 8 ? adam_mix(step->key + static_cast<uint32_t>(ch.tensor)) : 0;
  static_assert(kAdamChunk == kThreads * 4, "four values a thread");
  const int at = static_cast<int>(threadIdx.x) * 4;
  // whole waves leave together: encode() reduces over a wave
  if ((at & ~(kAdamBlock - 1)) >= left) return;
  const int64_t i = first + at;
  const int n = left - at >= 4 ? 4 : left - at > 0 ? static_cast<int>(left - at) : 0;
  float w[4], g[4], m[4], v[4];
  load4(t.w + i, n, w);
  load4(static_cast<const G*>(t.g) + i, n, g);
  if (pre != 1.f) {
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] *= pre;
  }
  if (BITS == 32) {
    load4(static_cast<const float*>(t.m) + i, n, m);
    load4(static_cast<const float*>(t.v) + i, n, v);
  } else {
    const int64_t b = i / kAdamBlock;
    decode(load_codes(static_cast<const uint8_t*>(t.m) + i, n), t.m_scale[b], m);
    decode(load_codes(static_cast<const uint8_t*>(t.v) + i, n), t.v_scale[b], v);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = v[j] * v[j];
  }
  float r[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float x = g[j] * f;
    m[j] = m[j] * b1 + x * c1;
    v[j] = v[j] * b2 + x * x * c2;
    r[j] = BITS == 32 ? sqrtf(v[j]) : root(v[j]);
  }
  uint32_t most_r = 0;
  if (BITS == 8) {
    if (n < 4) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j >= n) m[j] = v[j] = r[j] = 0.f;   // beyond the tensor: no part in the scale
    }
    most_r = wave_max(lane_most(r));
    if (most_r >= kInf || !__all(lane_least(r) >= __builtin_bit_cast(uint32_t, 0x1p-50f) - 1u)) {
#pragma unroll
      for (int j = 0; j < 4; ++j) r[j] = sqrtf(v[j]);
      most_r = wave_max(lane_most(r));
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = w[j] * keep - m[j] / (r[j] * ibc2 + eps) * rate;
  store4(t.w + i, n, w);
  if (t.low) {
    if (low_dtype == DBW_BF16)
      store4_half(static_cast<__bf16*>(t.low) + i, n, w);
    else
      store4_half(static_cast<_Float16*>(t.low) + i, n, w);
  }
  if (BITS == 32) {
    store4(static_cast<float*>(t.m) + i, n, m);
    store4(static_cast<float*>(t.v) + i, n, v);
  } else {
    uint32_t lo[4], hi[4];
    // (the indices of a lane start at a multiple of four: one product for all)
    const uint32_t at0 = adam_index(i) + key;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t u = adam_mix(at0 + adam_index(j));
      lo[j] = u << 16;
      hi[j] = u & 0xffff0000u;
    }
    uint32_t em, ev;
    const uint32_t cm = encode<false>(m, lo, wave_max(lane_most(m)), &em), cv = encode<true>(r, hi, most_r, &ev);
    store_codes(static_cast<uint8_t*>(t.m) + i, n, cm);
    store_codes(static_cast<uint8_t*>(t.v) + i, n, cv);
    if (threadIdx.x % 64 == 0) {
      const int64_t b = i / kAdamBlock;
      t.m_scale[b] = static_cast<uint8_t>(em);
      t.v_scale[b] = static_cast<uint8_t>(ev);
    }
  }
}

template <typename G>
hipError_t launch(const AdamArgs& a, hipStream_t s) {
  const bool norm = a.norm || a.h.max_norm > 0.0;
  const int64_t groups = (a.nchunks + kNormChunks - 1) / kNormChunks;
  const int parts = norm ? static_cast<int>(groups < kAdamNormParts ? groups : kAdamNormParts) : 0;
  if (parts) k_adamw_norm<G><<<parts, kThreads, 0, s>>>(a.tensors, a.chunks, a.nchunks, a.parts);
  k_adamw_prep<<<1, kThreads, 0, s>>>(a.step, a.parts, parts, a.h, a.norm);
  // (a launch holds fewer than 2^32 threads)
  constexpr int64_t kMost = int64_t{1} << 23;
  for (int64_t first = 0; first < a.nchunks; first += kMost) {
    const uint32_t grid = static_cast<uint32_t>(a.nchunks - first < kMost ? a.nchunks - first : kMost);
    if (a.bits == 8)
      k_adamw_update<G, 8><<<grid, kThreads, 0, s>>>(a.tensors, a.chunks + first, a.step, a.h, a.low_dtype);
    else
      k_adamw_update<G, 32><<<grid, kThreads, 0, s>>>(a.tensors, a.chunks + first, a.step, a.h, a.low_dtype);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_adamw(const AdamArgs& a, hipStream_t s) {
  if (a.g_dtype == DBW_F32) return launch<float>(a, s);
  if (a.g_dtype == DBW_BF16) return launch<__bf16>(a, s);
  return launch<_Float16>(a, s);
}

}  // namespace dbw
