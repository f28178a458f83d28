// Layer norm with its gradients, and the gradient of an activation with that
// of its bias.
//   k_norm         Y = (X - mean) / sqrt(var + eps) gamma + beta
//   k_norm_grad    dX, and each chunk's sums of dY H and dY
//   k_linear_grad  dZ = dY act'(Z), and each chunk's sums of dZ
//   k_chunk_sum    the weights' gradients of each group, from its chunks' sums
#include <hip/hip_runtime.h>

#include <algorithm>

#include "lm_ops.h"

namespace dbw {
namespace {

// Sixteen bytes of a row.
template <typename E>
struct Pack {
  static constexpr int N = 16 / sizeof(E);
  typedef E V __attribute__((ext_vector_type(N)));
  lm_u32x4 v;
  __device__ __forceinline__ float operator[](int j) const { return lm_to_f32(__builtin_bit_cast(V, v)[j]); }
};

// The columns of pack number p of a row of d values.  A row's last pack is its
// last N values: `skip` of them are the pack's before, which computes the same
// for them; sums leave them out.  Rows of fewer than N values are one pack.
template <int N>
struct Place {
  int base, skip, end;   // values [skip, end) are the pack's own
  __device__ __forceinline__ Place(int p, int d) {
    base = p * N;
    skip = 0;
    end = base < d ? N : 0;
    if (end && base + N > d) {
      if (d >= N) {
        skip = base + N - d;
        base = d - N;
      } else {
        end = d;
      }
    }
  }
  __device__ __forceinline__ bool own(int j) const { return j >= skip && j < end; }
  __device__ __forceinline__ bool whole() const { return skip == 0 && end == N; }
};

template <typename E>
__device__ __forceinline__ Pack<E> load(const E* row, const Place<Pack<E>::N>& p) {
  constexpr int N = Pack<E>::N;
  Pack<E> x;
  if (p.end == N) {
    x.v = *reinterpret_cast<const lm_u32x4_any*>(row + p.base);
  } else {
    typename Pack<E>::V v;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = j < p.end ? row[p.base + j] : static_cast<E>(0.f);
    x.v = __builtin_bit_cast(lm_u32x4, v);
  }
  return x;
}

template <typename E>
__device__ __forceinline__ void store(E* row, const Place<Pack<E>::N>& p, const float (&y)[Pack<E>::N]) {
  constexpr int N = Pack<E>::N;
  typedef float F __attribute__((ext_vector_type(N)));
  F f;
#pragma unroll
  for (int j = 0; j < N; ++j) f[j] = y[j];
  const typename Pack<E>::V v = __builtin_convertvector(f, typename Pack<E>::V);
  if (p.end == N) {
    *reinterpret_cast<lm_u32x4_any*>(row + p.base) = __builtin_bit_cast(lm_u32x4, v);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < p.end) row[p.base + j] = v[j];
  }
}

// N fp32 values from (to) p.base of a vector of weights.
template <int N>
__device__ __forceinline__ void load_f32(const float* w, const Place<N>& p, float (&x)[N]) {
  if (p.end == N) {
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      const lm_f32x4 v = *reinterpret_cast<const lm_f32x4_any*>(w + p.base + j);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[j + k] = v[k];
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = j < p.end ? w[p.base + j] : 0.f;
  }
}
template <int N>
__device__ __forceinline__ void store_f32(float* w, const Place<N>& p, const float (&x)[N]) {
  if (p.end == N) {
#pragma unroll
    for (int j = 0; j < N; j += 4)
      *reinterpret_cast<lm_f32x4_any*>(w + p.base + j) = lm_f32x4{x[j], x[j + 1], x[j + 2], x[j + 3]};
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < p.end) w[p.base + j] = x[j];
  }
}

// Sums of K values over a row's W waves; `turn` alternates the two halves of
// lds (2 K W floats), so that one barrier a sum is enough.
template <int W, int K>
__device__ __forceinline__ void row_sum(float (&v)[K], float* lds, int& turn) {
#pragma unroll
  for (int d = 32; d; d /= 2)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], d);
  if constexpr (W > 1) {
    float* mine = lds + turn * (K * W);
    turn ^= 1;
    if (threadIdx.x % 64 == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) mine[k * W + threadIdx.x / 64] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) v[k] += mine[k * W + w];
    }
  }
}

// Sums of f(j) over the pack's own values.
template <int N, typename F>
__device__ __forceinline__ void own_sum(const Place<N>& p, F f) {
  if (p.whole()) {
#pragma unroll
    for (int j = 0; j < N; ++j) f(j);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (p.own(j)) f(j);
  }
}

// W waves to a row, PACKS packs a thread.
template <typename E, int W, int PACKS>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_norm(NormArgs a) {
  constexpr int N = Pack<E>::N, TEAMS = W == 1 ? 4 : 1;
  __shared__ float lds[2 * 2 * W];
  const int tid = W == 1 ? threadIdx.x % 64 : threadIdx.x;
  const int64_t first = lm_offset(a.offsets, 0, a.T), end = lm_offset(a.offsets, a.n, a.T);
  const float over_d = 1.f / a.d;
  int turn = 0;
  for (int64_t t = first + static_cast<int64_t>(blockIdx.x) * TEAMS + (W == 1 ? threadIdx.x / 64 : 0); t < end;
       t += static_cast<int64_t>(gridDim.x) * TEAMS) {
    const E* row = static_cast<const E*>(a.X) + t * a.ld_X;
    Pack<E> x[PACKS];
    float sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < PACKS; ++i) {
      const Place<N> p(tid + i * W * 64, a.d);
      x[i] = load<E>(row, p);
      own_sum(p, [&](int j) { sum[0] += x[i][j]; });
    }
    row_sum<W, 1>(sum, lds, turn);
    const float mean = sum[0] * over_d;
    float sq[1] = {0.f};
#pragma unroll
    for (int i = 0; i < PACKS; ++i)
      own_sum(Place<N>(tid + i * W * 64, a.d), [&](int j) {
        const float c = x[i][j] - mean;
        sq[0] = fmaf(c, c, sq[0]);
      });
    row_sum<W, 1>(sq, lds, turn);
    const float r = 1.f / sqrtf(fmaf(sq[0], over_d, a.eps));
    E* out = static_cast<E*>(a.out) + t * a.ld_out;
#pragma unroll
    for (int i = 0; i < PACKS; ++i) {
      const Place<N> p(tid + i * W * 64, a.d);
      if (p.end == 0) continue;
      float g[N], b[N], y[N];
      load_f32<N>(a.gamma, p, g);
#pragma unroll
      for (int j = 0; j < N; ++j) b[j] = 0.f;
      if (a.beta) load_f32<N>(a.beta, p, b);
#pragma unroll
      for (int j = 0; j < N; ++j) y[j] = fmaf((x[i][j] - mean) * r, g[j], b[j]);
      store<E>(out, p, y);
    }
  }
}

template <typename E, int W, int PACKS>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_norm_grad(NormArgs a) {
  constexpr int N = Pack<E>::N, TEAMS = W == 1 ? 4 : 1;
  __shared__ float lds[2 * 3 * W];
  const int tid = W == 1 ? threadIdx.x % 64 : threadIdx.x;
  const uint32_t slot = blockIdx.x * TEAMS + (W == 1 ? threadIdx.x / 64 : 0);
  if (slot >= a.slots) return;
  const LmChunk chunk = lm_chunk(a.offsets, a.n, a.T, a.rows, slot, threadIdx.x % 64);
  const int64_t last = std::min<int64_t>(chunk.end, static_cast<int64_t>(chunk.first) + a.rows);
  if (chunk.empty()) return;
  const float over_d = 1.f / a.d;
  float dg[PACKS][N], db[PACKS][N];
#pragma unroll
  for (int i = 0; i < PACKS; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) dg[i][j] = db[i][j] = 0.f;
  int turn = 0;
  for (int64_t t = chunk.first; t < last; ++t) {
    const E* row = static_cast<const E*>(a.X) + t * a.ld_X;
    const E* grad = static_cast<const E*>(a.dY) + t * a.ld_dY;
    Pack<E> x[PACKS], dy[PACKS];
    float sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < PACKS; ++i) {
      const Place<N> p(tid + i * W * 64, a.d);
      x[i] = load<E>(row, p);
      dy[i] = load<E>(grad, p);
      own_sum(p, [&](int j) { sum[0] += x[i][j]; });
    }
    row_sum<W, 1>(sum, lds, turn);
    const float mean = sum[0] * over_d;
    // sums of (x - mean)^2, dH and dH (x - mean)
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < PACKS; ++i) {
      const Place<N> p(tid + i * W * 64, a.d);
      float g[N];
      load_f32<N>(a.gamma, p, g);
      own_sum(p, [&](int j) {
        const float c = x[i][j] - mean, h = dy[i][j] * g[j];
        s[0] = fmaf(c, c, s[0]);
        s[1] += h;
        s[2] = fmaf(h, c, s[2]);
      });
    }
    row_sum<W, 3>(s, lds, turn);
    const float r = 1.f / sqrtf(fmaf(s[0], over_d, a.eps));
    const float m1 = s[1] * over_d, m2 = s[2] * over_d * r;
    E* out = static_cast<E*>(a.out) + t * a.ld_out;
#pragma unroll
    for (int i = 0; i < PACKS; ++i) {
      const Place<N> p(tid + i * W * 64, a.d);
      if (p.end == 0) continue;
      float g[N], y[N];
      load_f32<N>(a.gamma, p, g);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float h = (x[i][j] - mean) * r, d = dy[i][j];
        dg[i][j] = fmaf(d, h, dg[i][j]);
        db[i][j] += d;
        y[j] = r * (fmaf(-h, m2, fmaf(d, g[j], -m1)));
      }
      store<E>(out, p, y);
    }
  }
  const int64_t ld = (a.d + 3) / 4 * 4;
  float* parts = a.parts + slot * ld;
#pragma unroll
  for (int i = 0; i < PACKS; ++i) {
    const Place<N> p(tid + i * W * 64, a.d);
    if (p.end == 0) continue;
    store_f32<N>(parts, p, dg[i]);
    if (a.dbeta) store_f32<N>(parts + a.slots * ld, p, db[i]);
  }
}

// A thread takes one pack of columns and every 256 / lanes-th row of its chunk.
template <typename E>
__global__ __launch_bounds__(256) void k_linear_grad(LinearGradArgs a, int lanes) {
  constexpr int N = Pack<E>::N;
  __shared__ float lds[256][N + 1];
  const uint32_t slot = blockIdx.x;
  const LmChunk chunk = lm_chunk(a.offsets, a.n, a.T, a.rows, slot, threadIdx.x % 64);
  if (chunk.empty()) return;
  const int64_t last = std::min<int64_t>(chunk.end, static_cast<int64_t>(chunk.first) + a.rows);
  const int step = 256 / lanes;
  const Place<N> p(static_cast<int>(blockIdx.y) * lanes + static_cast<int>(threadIdx.x) % lanes, a.C);
  float sum[N];
#pragma unroll
  for (int j = 0; j < N; ++j) sum[j] = 0.f;
  if (p.end)
    for (int64_t t = chunk.first + static_cast<int>(threadIdx.x) / lanes; t < last; t += step) {
      const Pack<E> dy = load<E>(static_cast<const E*>(a.dY) + t * a.ld_dY, p);
      float y[N];
#pragma unroll
      for (int j = 0; j < N; ++j) y[j] = dy[j];
      if (a.Z) {
        const Pack<E> z = load<E>(static_cast<const E*>(a.Z) + t * a.ld_Z, p);
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] *= lm_act_slope(z[j], a.act);
      }
      if (a.dZ) store<E>(static_cast<E*>(a.dZ) + t * a.ld_dZ, p, y);
#pragma unroll
      for (int j = 0; j < N; ++j) sum[j] += y[j];
    }
  if (!a.dbias) return;
  for (int s = 128; s >= lanes; s /= 2) {
    const int tid = threadIdx.x;
    if (tid >= s && tid < 2 * s)
#pragma unroll
      for (int j = 0; j < N; ++j) lds[tid][j] = sum[j];
    __syncthreads();
    if (tid < s)
#pragma unroll
      for (int j = 0; j < N; ++j) sum[j] += lds[tid + s][j];
  }
  if (static_cast<int>(threadIdx.x) < lanes && p.end) {
    const int64_t ld = (a.C + 3) / 4 * 4;
    store_f32<N>(a.parts + slot * ld, p, sum);
  }
}

// Sums of a group's chunks: 16 threads for four columns, each takes every 16th
// chunk.
struct ChunkSum {
  int n, d;
  int64_t T;
  const int32_t* offsets;
  uint32_t rows, slots;
  const float* parts;
  float* out[2];
  int64_t ld_out[2];
};
__global__ __launch_bounds__(256) void k_chunk_sum(ChunkSum a) {
  __shared__ lm_f32x4 lds[16][17];
  const int which = blockIdx.z, q = threadIdx.x % 16, part = threadIdx.x / 16;
  const int64_t ld = (a.d + 3) / 4 * 4;
  const uint32_t o0 = static_cast<uint32_t>(lm_offset(a.offsets, 0, a.T));
  for (int i = blockIdx.y; i < a.n; i += gridDim.y) {
    const int64_t first = lm_offset(a.offsets, i, a.T), end = lm_offset(a.offsets, i + 1, a.T);
    const uint32_t from = std::min(lm_first_slot(a.offsets, i, a.T, o0, a.rows), a.slots);
    const uint32_t count =
        end > first ? std::min(static_cast<uint32_t>((end - first + a.rows - 1) / a.rows), a.slots - from) : 0;
    const int c = (static_cast<int>(blockIdx.x) * 16 + q) * 4;
    lm_f32x4 x = {0.f, 0.f, 0.f, 0.f};
    if (c < a.d) {
      const float* p = a.parts + (static_cast<int64_t>(which) * a.slots + from) * ld + c;
#pragma unroll 8
      for (uint32_t s = part; s < count; s += 16) x += *reinterpret_cast<const lm_f32x4*>(p + s * ld);
    }
    lds[part][q] = x;
    __syncthreads();
    if (part == 0 && c < a.d) {
#pragma unroll
      for (int k = 1; k < 16; ++k) x += lds[k][q];
      float* out = a.out[which] + i * a.ld_out[which] + c;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c + j < a.d) out[j] = x[j];
    }
    __syncthreads();
  }
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int norm_waves(int d) { return d <= 1024 ? 1 : d <= 4096 ? 4 : 16; }

uint32_t norm_rows(int64_t T, int d) {
  const int w = norm_waves(d);
  const int64_t teams = w == 1 ? 4096 : w == 4 ? 1024 : 512;
  // (a launch holds fewer than 2^32 threads)
  return static_cast<uint32_t>(std::max({std::min<int64_t>(64, T / teams), int64_t{8}, T >> 21}));
}

int linear_lanes(int packs) {
  int lanes = 64;
  while (lanes > 1 && lanes / 2 >= packs) lanes /= 2;
  return lanes;
}

uint32_t linear_rows(int64_t T, int C) {
  const int64_t tiles = ceil_div(C, 512);
  return static_cast<uint32_t>(std::min<int64_t>(256, std::max<int64_t>(16, T * tiles / 1024)));
}

uint32_t slots_of(int n, int64_t T, uint32_t rows) { return static_cast<uint32_t>(T / rows + n); }

void launch_chunk_sum(const ChunkSum& c, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(ceil_div(c.d, 64)), std::min(c.n, 1024), c.out[1] ? 2 : 1);
  k_chunk_sum<<<grid, 256, 0, s>>>(c);
}

template <typename E, int W, int PACKS>
void norm_variant(const NormArgs& a, bool grad, hipStream_t s) {
  constexpr int TEAMS = W == 1 ? 4 : 1, THREADS = W == 1 ? 256 : 64 * W;
  if (grad) {
    k_norm_grad<E, W, PACKS><<<static_cast<uint32_t>(ceil_div(a.slots, TEAMS)), THREADS, 0, s>>>(a);
  } else {
    const int64_t most = W == 16 ? 1024 : 4096;
    k_norm<E, W, PACKS><<<static_cast<uint32_t>(std::min(most, ceil_div(a.T, TEAMS))), THREADS, 0, s>>>(a);
  }
}

template <typename E>
void norm_typed(const NormArgs& a, bool grad, hipStream_t s) {
  constexpr int N = Pack<E>::N;
  const int w = norm_waves(a.d);
  const int packs = static_cast<int>(ceil_div(a.d, N * 64 * w));
  if constexpr (N == 4) {
    if (packs > 2) {
      if (w == 1) return norm_variant<E, 1, 4>(a, grad, s);
      if (w == 4) return norm_variant<E, 4, 4>(a, grad, s);
      return norm_variant<E, 16, 4>(a, grad, s);
    }
  }
  if (w == 1) return packs > 1 ? norm_variant<E, 1, 2>(a, grad, s) : norm_variant<E, 1, 1>(a, grad, s);
  if (w == 4) return packs > 1 ? norm_variant<E, 4, 2>(a, grad, s) : norm_variant<E, 4, 1>(a, grad, s);
  return packs > 1 ? norm_variant<E, 16, 2>(a, grad, s) : norm_variant<E, 16, 1>(a, grad, s);
}

void norm(const NormArgs& a, bool grad, hipStream_t s) {
  if (a.dtype == DBW_F32) norm_typed<float>(a, grad, s);
  else if (a.dtype == DBW_BF16) norm_typed<__bf16>(a, grad, s);
  else norm_typed<_Float16>(a, grad, s);
}

}  // namespace

int64_t norm_workspace(int n, int64_t T, int d) {
  return int64_t{2} * 4 * slots_of(n, T, norm_rows(T, d)) * ((d + 3) / 4 * 4);
}

hipError_t launch_layer_norm(const NormArgs& a, hipStream_t s) {
  if (a.T == 0) return hipSuccess;
  norm(a, false, s);
  return hipGetLastError();
}

hipError_t launch_layer_norm_grad(NormArgs a, hipStream_t s) {
  a.rows = norm_rows(a.T, a.d);
  a.slots = slots_of(a.n, a.T, a.rows);
  if (a.T > 0) norm(a, true, s);
  launch_chunk_sum(ChunkSum{a.n, a.d, a.T, a.offsets, a.rows, a.slots, a.parts, {a.dgamma, a.dbeta},
                            {a.ld_dgamma, a.ld_dbeta}}, s);
  return hipGetLastError();
}

int64_t linear_grad_workspace(int n, int64_t T, int C) {
  return int64_t{4} * slots_of(n, T, linear_rows(T, C)) * ((C + 3) / 4 * 4);
}

hipError_t launch_linear_grad(LinearGradArgs a, hipStream_t s) {
  a.rows = linear_rows(a.T, a.C);
  a.slots = slots_of(a.n, a.T, a.rows);
  if (a.T > 0) {
    const int packs = static_cast<int>(ceil_div(a.C, a.dtype == DBW_F32 ? 4 : 8));
    const int lanes = linear_lanes(packs);
    const dim3 grid(a.slots, static_cast<uint32_t>(ceil_div(packs, lanes)));
    if (a.dtype == DBW_F32) k_linear_grad<float><<<grid, 256, 0, s>>>(a, lanes);
    else if (a.dtype == DBW_BF16) k_linear_grad<__bf16><<<grid, 256, 0, s>>>(a, lanes);
    else k_linear_grad<_Float16><<<grid, 256, 0, s>>>(a, lanes);
  }
  if (a.dbias)
    launch_chunk_sum(ChunkSum{a.n, a.C, a.T, a.offsets, a.rows, a.slots, a.parts, {a.dbias, nullptr}, {a.ld_dbias, 0}}, s);
  return hipGetLastError();
}

}  // namespace dbw
