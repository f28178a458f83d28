// Token loss: mean cross entropy of each worker's rows, and its gradient.
//   k_token_count  live rows of each worker -> 1 / count
//   k_token_rows   a workgroup (or a wave) to a row: loss and gradient
//   k_token_mean   a workgroup to a worker: the mean of its rows' losses
//
// k_token_rows is bound by memory: T C logits read once and as many gradients
// written once.  A row stays in registers, as it was loaded, between the
// maximum, the sum of exponentials and the gradient; each of the three
// evaluates what it needs from there (the exponentials twice: 2 of the some 12
// operations a value, against a second read of the row).  Rows beyond what a
// workgroup's registers hold are read a second time.
//
// softmax(z)_c = exp(z_c - max) / sum exp(z - max), in fp32.  The maximum is
// subtracted before the product with log2(e), which could overflow.
#include <hip/hip_runtime.h>

#include <cmath>

#include "lm_ops.h"

namespace dbw {
namespace {

constexpr int64_t kMaxGrid = int64_t{1} << 20;
constexpr float kLog2e = 1.44269504088896341f;

__global__ __launch_bounds__(256) void k_token_count(int n, int64_t T, const int32_t* __restrict__ offsets,
                                                     const int32_t* __restrict__ y, float* __restrict__ inv) {
  const int i = blockIdx.x;
  const int64_t a = lm_offset(offsets, i, T), b = lm_offset(offsets, i + 1, T);
  int count = 0;
  for (int64_t t = a + threadIdx.x; t < b; t += 256) count += y[t] >= 0;
#pragma unroll
  for (int d = 32; d; d /= 2) count += __shfl_xor(count, d);
  __shared__ int waves[4];
  if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = count;
  __syncthreads();
  if (threadIdx.x == 0) {
    const int all = waves[0] + waves[1] + waves[2] + waves[3];
    inv[i] = all ? static_cast<float>(1.0 / all) : 0.f;
  }
}

__global__ __launch_bounds__(256) void k_token_mean(int n, int64_t T, const int32_t* __restrict__ offsets,
                                                    const float* __restrict__ row_loss, const int32_t* __restrict__ y,
                                                    float* __restrict__ loss) {
  const int i = blockIdx.x;
  const int64_t a = lm_offset(offsets, i, T), b = lm_offset(offsets, i + 1, T);
  double sum = 0.0;
  int count = 0;
  for (int64_t t = a + threadIdx.x; t < b; t += 256) {
    const bool live = y[t] >= 0;
    count += live;
    sum += live ? row_loss[t] : 0.f;
  }
#pragma unroll
  for (int d = 32; d; d /= 2) {
    sum += __shfl_xor(sum, d);
    count += __shfl_xor(count, d);
  }
  __shared__ double sums[4];
  __shared__ int counts[4];
  if (threadIdx.x % 64 == 0) {
    sums[threadIdx.x / 64] = sum;
    counts[threadIdx.x / 64] = count;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const int all = counts[0] + counts[1] + counts[2] + counts[3];
    loss[i] = all ? static_cast<float>(((sums[0] + sums[1]) + (sums[2] + sums[3])) / all) : 0.f;
  }
}

// Sixteen bytes of logits.
template <typename E>
struct Pack {
  static constexpr int N = 16 / sizeof(E);
  typedef E V __attribute__((ext_vector_type(16 / sizeof(E))));
};

template <typename E>
__device__ __forceinline__ lm_u32x4 load_pack(const E* p, int64_t n, E fill) {
  if (n >= Pack<E>::N) return *reinterpret_cast<const lm_u32x4_any*>(p);
  typename Pack<E>::V v;
#pragma unroll
  for (int j = 0; j < Pack<E>::N; ++j) v[j] = j < n ? p[j] : fill;
  return __builtin_bit_cast(lm_u32x4, v);
}
template <typename E>
__device__ __forceinline__ void store_pack(E* p, int64_t n, typename Pack<E>::V v) {
  if (n >= Pack<E>::N) {
    *reinterpret_cast<lm_u32x4_any*>(p) = __builtin_bit_cast(lm_u32x4, v);
  } else {
#pragma unroll
    for (int j = 0; j < Pack<E>::N; ++j)
      if (j < n) p[j] = v[j];
  }
}

template <int THREADS>
__device__ __forceinline__ float row_max(float v, float* lds) {
  // a NaN has to survive: fmaxf drops it, the sum of exponentials brings it back
#pragma unroll
  for (int d = 32; d; d /= 2) v = fmaxf(v, __shfl_xor(v, d));
  if (THREADS == 64) return v;
  __syncthreads();
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int i = 1; i < THREADS / 64; ++i) v = fmaxf(v, lds[i]);
  return v;
}
template <int THREADS>
__device__ __forceinline__ float row_sum(float v, float* lds) {
#pragma unroll
  for (int d = 32; d; d /= 2) v += __shfl_xor(v, d);
  if (THREADS == 64) return v;
  __syncthreads();
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int i = 1; i < THREADS / 64; ++i) v += lds[i];
  return v;
}

// One row by THREADS threads, PACKS packs of 16 bytes a thread held in
// registers; PACKS = 0: the row is read twice.
template <typename E, int THREADS, int PACKS>
__device__ __forceinline__ void token_row(const TokenArgs& a, int64_t t, int tid, float* lds) {
  constexpr int N = Pack<E>::N;
  typedef typename Pack<E>::V V;
  // the worker of the row: how many of offsets[1..n] are at most t
  if (t < lm_offset(a.offsets, 0, a.T)) return;
  int worker = 0;
  for (int i = threadIdx.x % 64; i < a.n; i += 64) worker += lm_offset(a.offsets, i + 1, a.T) <= t;
#pragma unroll
  for (int d = 32; d; d /= 2) worker += __shfl_xor(worker, d);
  if (worker >= a.n) return;

  const E* z = static_cast<const E*>(a.Z) + t * a.ld_Z;
  E* dz = a.dZ ? static_cast<E*>(a.dZ) + t * a.ld_dZ : nullptr;
  const int y = a.y[t];
  const int C = a.C;
  if (y < 0) {
    if (dz) {
      V zero;
#pragma unroll
      for (int j = 0; j < N; ++j) zero[j] = static_cast<E>(0.f);
      for (int c = tid * N; c < C; c += THREADS * N) store_pack<E>(dz + c, C - c, zero);
    }
    return;
  }
  const E low = static_cast<E>(-INFINITY);
  const float zy = y < C ? lm_to_f32(z[y]) : NAN;   // read before any store: dZ may be Z
  float top = -INFINITY, sum = 0.f;
  lm_u32x4 held[PACKS ? PACKS : 1];
  if (PACKS) {
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      const int c = (p * THREADS + tid) * N;
      if (c < C) {
        held[p] = load_pack<E>(z + c, C - c, low);
      } else {
        V v;
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = low;
        held[p] = __builtin_bit_cast(lm_u32x4, v);
      }
    }
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      const V v = __builtin_bit_cast(V, held[p]);
#pragma unroll
      for (int j = 0; j < N; ++j) top = fmaxf(top, lm_to_f32(v[j]));
    }
    top = row_max<THREADS>(top, lds);
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      const V v = __builtin_bit_cast(V, held[p]);
#pragma unroll
      for (int j = 0; j < N; ++j) sum += __builtin_amdgcn_exp2f((lm_to_f32(v[j]) - top) * kLog2e);
    }
    sum = row_sum<THREADS>(sum, lds);
  } else {
    // running maximum and sum of every thread, joined at the end
    float mx = -INFINITY;
    for (int c = tid * N; c < C; c += THREADS * N) {
      const V v = __builtin_bit_cast(V, load_pack<E>(z + c, C - c, low));
      float m = mx;
#pragma unroll
      for (int j = 0; j < N; ++j) m = fmaxf(m, lm_to_f32(v[j]));
      // a thread that has seen only -infinities keeps 0 (NaNs pass)
      sum = m == mx ? sum : sum * __builtin_amdgcn_exp2f((mx - m) * kLog2e);
      mx = m;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float x = lm_to_f32(v[j]);
        sum += x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((x - m) * kLog2e);
      }
    }
    top = row_max<THREADS>(mx, lds);
    sum = mx == -INFINITY && sum == 0.f && top != -INFINITY ? 0.f
                                                              : sum * __builtin_amdgcn_exp2f((mx - top) * kLog2e);
    sum = row_sum<THREADS>(sum, lds);
  }
  if (tid == 0) a.row_loss[t] = logf(sum) + (top - zy);
  if (!dz) return;
  const float s = a.scale * a.inv[worker];
  const float f = y < C ? s / sum : NAN;
  if (PACKS) {
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      const int c = (p * THREADS + tid) * N;
      if (c < C) {
        const V v = __builtin_bit_cast(V, held[p]);
        V o;
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float e = __builtin_amdgcn_exp2f((lm_to_f32(v[j]) - top) * kLog2e);
          o[j] = static_cast<E>(e * f - (c + j == y ? s : 0.f));
        }
        store_pack<E>(dz + c, C - c, o);
      }
    }
  } else {
    for (int c = tid * N; c < C; c += THREADS * N) {
      const V v = __builtin_bit_cast(V, load_pack<E>(z + c, C - c, low));
      V o;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float e = __builtin_amdgcn_exp2f((lm_to_f32(v[j]) - top) * kLog2e);
        o[j] = static_cast<E>(e * f - (c + j == y ? s : 0.f));
      }
      store_pack<E>(dz + c, C - c, o);
    }
  }
}

template <typename E, int THREADS, int PACKS>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void k_token_rows(TokenArgs a) {
  __shared__ float lds[THREADS / 64];
  const int tid = THREADS == 64 ? threadIdx.x % 64 : threadIdx.x;
  constexpr int ROWS = THREADS == 64 ? 4 : 1;   // rows of a workgroup
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * ROWS + (ROWS > 1 ? threadIdx.x / 64 : 0); t < a.T;
       t += static_cast<int64_t>(gridDim.x) * ROWS)
    token_row<E, THREADS, PACKS>(a, t, tid, lds);
}

template <typename E>
void launch_rows(const TokenArgs& a, hipStream_t s) {
  constexpr int N = Pack<E>::N;
  const int64_t packs = (a.C + N - 1) / N;
  // (a launch holds fewer than 2^32 threads: the kernel goes over the rest)
  const uint32_t T = static_cast<uint32_t>(a.T < kMaxGrid ? a.T : kMaxGrid);
  if (packs <= 64 * 8)
    k_token_rows<E, 64, 8><<<(T + 3) / 4, 256, 0, s>>>(a);
  else if (packs <= 256 * 8)
    k_token_rows<E, 256, 8><<<T, 256, 0, s>>>(a);
  else if (packs <= 1024 * 8)
    k_token_rows<E, 1024, 8><<<T, 1024, 0, s>>>(a);
  else
    k_token_rows<E, 1024, 0><<<T, 1024, 0, s>>>(a);
}

}  // namespace

hipError_t launch_token_loss(const TokenArgs& a, hipStream_t s) {
  if (a.dZ) k_token_count<<<a.n, 256, 0, s>>>(a.n, a.T, a.offsets, a.y, a.inv);
  if (a.T) {
    if (a.dtype == DBW_F32)
      launch_rows<float>(a, s);
    else if (a.dtype == DBW_BF16)
      launch_rows<__bf16>(a, s);
    else
      launch_rows<_Float16>(a, s);
  }
  k_token_mean<<<a.n, 256, 0, s>>>(a.n, a.T, a.offsets, a.row_loss, a.y, a.loss);
  return hipGetLastError();
}

}  // namespace dbw
