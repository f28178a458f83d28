// Token loss: mean cross entropy of each worker's rows, and its gradient.
//   k_token_count  live rows of each worker, in parts (few rows: counted by
//                  k_token_rows itself)
//   k_token_rows   a workgroup (or a wave) to a row: loss and gradient
//   k_token_sum    sums of the workers' row losses, in parts (many rows only)
//   k_token_mean   a workgroup to a worker: the mean
//
// k_token_rows is bound by memory: T C logits read once and as many gradients
// written once.  A row stays in registers, as it was loaded, between the
// maximum, the sum of exponentials and the gradient; each of the three
// evaluates what it needs from there (the exponentials twice: 2 of the some 12
// operations a value, against a second read of the row).  Rows beyond what a
// workgroup's registers hold are read a second time.
//
// A row takes as few threads as hold it in 16 packs each, so that two or more
// workgroups share a CU and one's exponentials run beside another's loads and
// stores: 8192 x 50257 bf16 330 us, 5.0 TB/s (a large copy reaches 4.9), where 1024
// threads of 8 packs, alone on a CU, took 542.  Rows of up to 131072 16-bit
// values fill a CU by themselves (2048 x 128000 fp16 233 us, 4.5 TB/s), longer ones
// are read twice (1024 x 200000 bf16 233 us, 3.5 TB/s by their size).
//
// softmax(z)_c = 2^(b (z_c - max)) / sum 2^(b (z - max)) with b = log2(e), in
// fp32.  The difference comes first where that costs nothing: it is 0 at the
// maximum, whatever its size.  16-bit rows held in registers take 2^(b z - b max)
// instead, one fused multiply-add for two operations (2048 x 128000 fp16 246 us
// for 265, 8192 x 50257 bf16 345 for 356; 4096 x 32000 fp32 203 for 202).  There b
// max is rounded; that factor is the same above and below, and is taken out of
// the loss.  It is at most 2 below |max| = 2^24, but would be beyond every
// exponent from 2^31 on: see HalfPower.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "lm_ops.h"

namespace dbw {
namespace {

constexpr int64_t kMaxGrid = int64_t{1} << 20;
constexpr float kLog2e = 1.44269504088896341f;

// Rows [a, b) of part `part` of the rows of worker i.
__device__ __forceinline__ void part_rows(const TokenArgs& g, int i, int part, int64_t* a, int64_t* b) {
  const int64_t first = lm_offset(g.offsets, i, g.T), end = lm_offset(g.offsets, i + 1, g.T);
  const int64_t all = end > first ? end - first : 0, each = (all + g.parts - 1) / g.parts;
  *a = first + (part * each < all ? part * each : all);
  *b = first + ((part + 1) * each < all ? (part + 1) * each : all);
}

__device__ __forceinline__ int wave_sum(int v) {
#pragma unroll
  for (int d = 32; d; d /= 2) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 32; d; d /= 2) v += __shfl_xor(v, d);
  return v;
}

__global__ __launch_bounds__(256) void k_token_count(TokenArgs g) {
  const int i = blockIdx.x / g.parts, part = blockIdx.x % g.parts;
  int64_t a, b;
  part_rows(g, i, part, &a, &b);
  int count = 0;
#pragma unroll 4
  for (int64_t t = a + threadIdx.x; t < b; t += 256) count += g.y[t] >= 0;
  count = wave_sum(count);
  __shared__ int waves[4];
  if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = count;
  __syncthreads();
  if (threadIdx.x == 0) g.counts[blockIdx.x] = waves[0] + waves[1] + waves[2] + waves[3];
}

// Sum and number of the live rows [a, b), for thread 0 (in a fixed order).
__device__ __forceinline__ void sum_rows(const TokenArgs& g, int64_t a, int64_t b, double* all, int* live) {
  double sum = 0.0;
  int count = 0;
#pragma unroll 4
  for (int64_t t = a + threadIdx.x; t < b; t += 256) {
    const bool is = g.y[t] >= 0;
    count += is;
    sum += is ? g.row_loss[t] : 0.f;
  }
  sum = wave_sum(sum);
  count = wave_sum(count);
  __shared__ double sums[4];
  __shared__ int counts[4];
  if (threadIdx.x % 64 == 0) {
    sums[threadIdx.x / 64] = sum;
    counts[threadIdx.x / 64] = count;
  }
  __syncthreads();
  *all = (sums[0] + sums[1]) + (sums[2] + sums[3]);
  *live = counts[0] + counts[1] + counts[2] + counts[3];
}

__global__ __launch_bounds__(256) void k_token_sum(TokenArgs g) {
  int64_t a, b;
  part_rows(g, blockIdx.x / g.parts, blockIdx.x % g.parts, &a, &b);
  double sum;
  int count;
  sum_rows(g, a, b, &sum, &count);
  if (threadIdx.x == 0) {
    g.sums[blockIdx.x] = sum;
    g.counts[blockIdx.x] = count;
  }
}

__global__ __launch_bounds__(256) void k_token_mean(TokenArgs g) {
  const int i = blockIdx.x;
  double sum = 0.0;
  int count = 0;
  if (g.parts > 1) {
    for (int p = 0; p < g.parts; ++p) {
      sum += g.sums[i * g.parts + p];
      count += g.counts[i * g.parts + p];
    }
  } else {
    int64_t a, b;
    part_rows(g, i, 0, &a, &b);
    sum_rows(g, a, b, &sum, &count);
  }
  if (threadIdx.x == 0) g.loss[i] = count ? static_cast<float>(sum / count) : 0.f;
}

// Sixteen bytes of logits.
template <typename E>
struct Pack {
  static constexpr int N = 16 / sizeof(E);
  typedef E V __attribute__((ext_vector_type(16 / sizeof(E))));
};

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

// e^(x - max): 0 where the difference is infinite, NaN for two infinities of
// one sign.
struct Power {
  float max;
  __device__ __forceinline__ explicit Power(float m) : max(m) {}
  __device__ __forceinline__ float operator()(float x) const { return __builtin_amdgcn_exp2f((x - max) * kLog2e); }
  __device__ __forceinline__ float lost() const { return 0.f; }
};
// The same of 16-bit values, times a factor that all of a row share and whose
// logarithm is lost().  From |max| = 2^24 on, bf16 values below max are 2^16 or
// more below it: their powers are 0 to any base, and with b = 1 nothing is
// rounded.
struct HalfPower {
  float b, bm, max;
  __device__ __forceinline__ explicit HalfPower(float m) : max(m) {
#pragma clang fp contract(off)   // bm is the rounded product wherever it is used
    b = fabsf(m) < 0x1p24f ? kLog2e : 1.f;
    bm = b * m;
  }
  __device__ __forceinline__ float operator()(float x) const { return __builtin_amdgcn_exp2f(fmaf(x, b, -bm)); }
  __device__ __forceinline__ float lost() const { return fmaf(max, b, -bm) * 0.693147180559945309f; }
};

// One row by THREADS threads, PACKS packs of 16 bytes a thread held in
// registers; PACKS = 0: the row is read twice.
template <typename E, int THREADS, int PACKS>
__device__ __forceinline__ void token_row(const TokenArgs& a, int64_t t, int tid, float* lds) {
  constexpr int N = Pack<E>::N;
  typedef typename Pack<E>::V V;
  const int lane = threadIdx.x % 64;
  // the worker of the row: how many of offsets[1..n] are at most t
  if (t < lm_offset(a.offsets, 0, a.T)) return;
  int worker = 0;
  for (int i = lane; i < a.n; i += 64) worker += lm_offset(a.offsets, i + 1, a.T) <= t;
  worker = wave_sum(worker);
  if (worker >= a.n) return;

  const E* z = static_cast<const E*>(a.Z) + t * a.ld_Z;
  E* dz = a.dZ ? static_cast<E*>(a.dZ) + t * a.ld_dZ : nullptr;
  const int y = a.y[t];
  const int C = a.C;
  // the row in whole packs at whole 16 bytes of memory, and the values before
  // and behind them, one a thread
  const int off = static_cast<int>(reinterpret_cast<uintptr_t>(z) % 16 / sizeof(E));
  const int head = off ? (N - off < C ? N - off : C) : 0;
  const int packs = (C - head) / N;
  const int edge = tid < head ? tid : head + packs * N + tid - head;
  const bool has_edge = tid < head || (tid < 2 * N && edge < C);
  const E* zb = z + head;
  E* db = dz + head;
  if (y < 0) {
    if (dz) {
      for (int p = tid; p < packs; p += THREADS) *reinterpret_cast<lm_u32x4_any*>(db + p * N) = lm_u32x4{0, 0, 0, 0};
      if (has_edge) dz[edge] = static_cast<E>(0.f);
    }
    return;
  }
  const E low = static_cast<E>(-INFINITY);
  const float zy = y < C ? lm_to_f32(z[y]) : NAN;   // read before any store: dZ may be Z
  const float ze = has_edge ? lm_to_f32(z[edge]) : -INFINITY;
  typedef std::conditional_t<PACKS && sizeof(E) == 2, HalfPower, Power> P;
  float top, sum;
  lm_u32x4 held[PACKS ? PACKS : 1];
  if (PACKS) {
    V fill;
#pragma unroll
    for (int j = 0; j < N; ++j) fill[j] = low;
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      held[p] = __builtin_bit_cast(lm_u32x4, fill);
      if (p * THREADS + tid < packs) held[p] = *reinterpret_cast<const lm_u32x4_any*>(zb + (p * THREADS + tid) * N);
    }
    top = ze;
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      const V v = __builtin_bit_cast(V, held[p]);
#pragma unroll
      for (int j = 0; j < N; ++j) top = fmaxf(top, lm_to_f32(v[j]));
    }
    top = row_max<THREADS>(top, lds);
    const P e(top);
    sum = e(ze);
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      asm volatile("" : "+v"(held[p]));   // unpacked anew: the values are not kept as fp32
      const V v = __builtin_bit_cast(V, held[p]);
#pragma unroll
      for (int j = 0; j < N; ++j) sum += e(lm_to_f32(v[j]));
    }
    sum = row_sum<THREADS>(sum, lds);
  } else {
    // running maximum and sum of every thread, joined at the end; a thread
    // that has seen only -infinities keeps 0
    float mx = ze;
    sum = ze == -INFINITY ? 0.f : Power(mx)(ze);
    for (int p = tid; p < packs; p += THREADS) {
      const V v = __builtin_bit_cast(V, static_cast<lm_u32x4>(*reinterpret_cast<const lm_u32x4_any*>(zb + p * N)));
      float m = mx;
#pragma unroll
      for (int j = 0; j < N; ++j) m = fmaxf(m, lm_to_f32(v[j]));
      if (m != mx) {
        sum *= Power(m)(mx);
        mx = m;
      }
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float x = lm_to_f32(v[j]);
        sum += x == -INFINITY ? 0.f : Power(mx)(x);
      }
    }
    top = row_max<THREADS>(mx, lds);
    sum *= Power(top)(mx);
    sum = row_sum<THREADS>(sum, lds);
  }
  const P e(top);
  if (tid == 0) a.row_loss[t] = logf(sum) - e.lost() + (top - zy);
  if (!dz) return;
  // live rows of the worker (at least this one)
  int count = 0;
  if (a.parts == 0) {
    const int64_t end = lm_offset(a.offsets, worker + 1, a.T);
    for (int64_t r = lm_offset(a.offsets, worker, a.T) + lane; r < end; r += 64) count += a.y[r] >= 0;
  } else if (lane < a.parts) {
    count = a.counts[worker * a.parts + lane];
  }
  const float s = a.scale / static_cast<float>(wave_sum(count));
  const float f = y < C ? s / sum : NAN;
  if (has_edge) dz[edge] = static_cast<E>(e(ze) * f - (edge == y ? s : 0.f));
  const auto gradient = [&](const lm_u32x4& x, int p) {
    const V v = __builtin_bit_cast(V, x);
    const int at = y - head - p * N;
    V o;
#pragma unroll
    for (int j = 0; j < N; ++j) o[j] = static_cast<E>(e(lm_to_f32(v[j])) * f);
    *reinterpret_cast<lm_u32x4_any*>(db + p * N) = __builtin_bit_cast(lm_u32x4, o);
    if (at >= 0 && at < N) dz[y] = static_cast<E>(e(zy) * f - s);   // (after its pack, by the same thread)
  };
  if (PACKS) {
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      asm volatile("" : "+v"(held[p]));
      if (p * THREADS + tid < packs) gradient(held[p], p * THREADS + tid);
    }
  } else {
    for (int p = tid; p < packs; p += THREADS)
      gradient(static_cast<lm_u32x4>(*reinterpret_cast<const lm_u32x4_any*>(zb + p * N)), p);
  }
}

// THREADS to a row (64: four rows to a workgroup).  A held pack takes four
// registers: as many waves as leave that room without spilling, so that
// workgroups load, compute and store beside each other.
template <typename E, int THREADS, int PACKS>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS, PACKS <= 4 ? 8 : PACKS <= 8 ? 5 : 4) void k_token_rows(
    TokenArgs a) {
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
  const int64_t packs = a.C / N;   // at most, by where the row starts
  // (a launch holds fewer than 2^32 threads: the kernel goes over the rest)
  const uint32_t T = static_cast<uint32_t>(std::min(a.T, kMaxGrid));
  if (packs <= 64 * 2)
    k_token_rows<E, 64, 2><<<(T + 3) / 4, 256, 0, s>>>(a);
  else if (packs <= 64 * 8)
    k_token_rows<E, 64, 8><<<(T + 3) / 4, 256, 0, s>>>(a);
  else if (packs <= 256 * 4)
    k_token_rows<E, 256, 4><<<T, 256, 0, s>>>(a);
  else if (packs <= 256 * 8)
    k_token_rows<E, 256, 8><<<T, 256, 0, s>>>(a);
  else if (packs <= 256 * 16)
    k_token_rows<E, 256, 16><<<T, 256, 0, s>>>(a);
  else if (packs <= 512 * 16)
    k_token_rows<E, 512, 16><<<T, 512, 0, s>>>(a);
  else if (packs <= 1024 * 16)
    k_token_rows<E, 1024, 16><<<T, 1024, 0, s>>>(a);
  else
    k_token_rows<E, 1024, 0><<<T, 1024, 0, s>>>(a);
}

}  // namespace

hipError_t launch_token_loss(const TokenArgs& args, hipStream_t s) {
  TokenArgs a = args;
  // Parts by all rows, not by a worker's even share, as one may have them all:
  // 65536 x 100 bf16, 16 workers, all rows to one, 145 us in one part and 58 in
  // several (evenly shared 49 and 45).  At most 4096 parts in all: 900 workers pay
  // 4 to 7 us for four parts when they share evenly (65536 rows 64 and 70) and
  // save 67 when one has all (166 and 99).  A second part costs a launch: 16384
  // rows of 16 workers 21 us for 19 evenly shared, 31 for 40 all to one; hence
  // none up to 8192 rows, but for a worker that has them all for certain (8192
  // rows 21 us for 25).  Up to 1024 rows in all, a row's wave counts its
  // worker's labels itself (16 loads a lane) and saves a launch.
  const int64_t most = std::min<int64_t>(kTokenParts, std::max(1, 4096 / a.n));
  const int64_t parts = 1 + (a.n == 1 ? a.T : a.T - 1) / 8192;
  a.parts = a.T <= 1024 ? 0 : static_cast<int>(std::min<int64_t>(most, parts));
  if (a.dZ && a.parts) k_token_count<<<a.n * a.parts, 256, 0, s>>>(a);
  if (a.T) {
    if (a.dtype == DBW_F32)
      launch_rows<float>(a, s);
    else if (a.dtype == DBW_BF16)
      launch_rows<__bf16>(a, s);
    else
      launch_rows<_Float16>(a, s);
  }
  a.parts = std::max(a.parts, 1);
  if (a.parts > 1) k_token_sum<<<a.n * a.parts, 256, 0, s>>>(a);
  k_token_mean<<<a.n, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace dbw
