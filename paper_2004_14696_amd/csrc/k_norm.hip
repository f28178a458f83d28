// Layer norm with its gradients, and the gradient of an activation with that
// of its bias.
//   k_norm         Y = (X - mean) / sqrt(var + eps) gamma + beta
//   k_norm_grad    dX, and sums of dY H and dY over pieces of the groups
//   k_linear_grad  dZ = dY act'(Z), and sums of dZ over pieces
//   k_piece_sum    the weights' gradients of each group, from its pieces' sums
//
// The rows of all groups are dealt out evenly, in parts; where a group ends
// inside a part, its piece ends.
//
// All are bound by memory, each array read or written once.  A row stays in
// registers from its load to the result, the next one is on its way meanwhile;
// mean, variance and the two sums of dH take two reductions over its waves.
// us, and TB/s of the arrays' bytes (a large copy reaches 5.1 to 5.2): forward
// 16384 x 4096 bf16 56, 4.8 (4090 columns 55); 8192 x 8192 bf16 51, 5.3; 4096 x 16384 fp32
// 99, 5.4; gradients with the sums over pieces 8192 x 4096 bf16 58, 3.5 (the sums of
// 768 parts written and read, 50 MB, are not in the rate); 3001 x 1003 fp32 of 64 groups
// 19, four launch latencies long; linear gradient 8192 x 4096 bf16, GELU, 49, 4.1.
// A branch around the loads of packs behind a row's end made each wait for the
// one before (gradients 3001 x 1003 17 us for 13); masks of every pack, where only a
// row's last can need one, filled the registers (16384 x 4090 forward 89 and 165 us).
// Gradients of the widest rows do not fit them and spill: 4 packs for 16 waves in
// fp32 (21 registers; 4096 x 16384 240 us, 3.4 TB/s, x 12288 147, 4.1; odd widths 36, x 16383
// 322 us), 2 packs of 16-bit values in odd widths (19; 8192 x 16380 bf16 315 us, x 16384
// 199).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "lm_ops.h"

namespace dbw {
namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Sixteen bytes of a row.
template <typename E>
struct Pack {
  static constexpr int N = 16 / sizeof(E);
  typedef E V __attribute__((ext_vector_type(N)));
  lm_u32x4 v;
  __device__ __forceinline__ float operator[](int j) const { return lm_to_f32(__builtin_bit_cast(V, v)[j]); }
};

// The columns of pack number p of a row of d values.  A row's last pack is its
// last N values: the first of them may be the pack's before, which computes the
// same for them; sums over a row leave them out.  Rows of fewer than N values are
// one pack.  WHOLE: d is a multiple of N.  Only where `last` is true may the pack
// be the row's last one, or behind it.
template <int N, bool WHOLE = false>
struct Place {
  int base, end;   // `end` values from base on
  uint32_t mask;   // those of them that are the pack's own
  bool wide;       // rows have N values at least
  __device__ __forceinline__ Place(int p, int d, bool last = true) : base(p * N), end(N), wide(true) {
    int skip = 0;
    if (last) {
      wide = WHOLE || d >= N;
      end = base < d ? N : 0;
      if (!WHOLE && end && base + N > d) {
        if (d >= N) {
          skip = base + N - d;
          base = d - N;
        } else {
          end = d;
        }
      }
    }
    mask = (1u << end) - (1u << skip);
  }
  // 1 for values of the pack's own: a factor, which costs less than a branch
  __device__ __forceinline__ float own(int j) const {
    return WHOLE ? 1.f : __builtin_bit_cast(float, static_cast<uint32_t>(static_cast<int32_t>(mask << (31 - j)) >> 31) & 0x3f800000u);
  }
  __device__ __forceinline__ bool full() const { return WHOLE || end == N; }
  __device__ __forceinline__ bool vectors() const { return wide; }
};

// Loads are the same for packs behind the row's end, which read its start and
// get zeros: a branch around each would make them wait for one another.
template <typename E, typename P>
__device__ __forceinline__ Pack<E> load(const E* row, const P& p) {
  constexpr int N = Pack<E>::N;
  Pack<E> x;
  if (p.vectors()) {
    const lm_u32x4 v = *reinterpret_cast<const lm_u32x4_any*>(row + (p.end ? p.base : 0));
    x.v = p.end ? v : lm_u32x4{0, 0, 0, 0};
  } else {
    typename Pack<E>::V v;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = j < p.end ? row[p.base + j] : static_cast<E>(0.f);
    x.v = __builtin_bit_cast(lm_u32x4, v);
  }
  return x;
}

template <typename E, typename P>
__device__ __forceinline__ void store(E* row, const P& p, const float (&y)[Pack<E>::N]) {
  constexpr int N = Pack<E>::N;
  typedef float F __attribute__((ext_vector_type(N)));
  F f;
#pragma unroll
  for (int j = 0; j < N; ++j) f[j] = y[j];
  const typename Pack<E>::V v = __builtin_convertvector(f, typename Pack<E>::V);
  if (p.full()) {
    *reinterpret_cast<lm_u32x4_any*>(row + p.base) = __builtin_bit_cast(lm_u32x4, v);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < p.end) row[p.base + j] = v[j];
  }
}

// N fp32 values from (to) p.base of a vector of weights.
template <int N, typename P>
__device__ __forceinline__ void load_f32(const float* w, const P& p, float (&x)[N]) {
  if (p.vectors()) {
    const float* at = w + (p.end ? p.base : 0);
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      const lm_f32x4 v = *reinterpret_cast<const lm_f32x4_any*>(at + j);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[j + k] = v[k];
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = j < p.end ? w[p.base + j] : 0.f;
  }
}
template <int N, typename P>
__device__ __forceinline__ void store_f32(float* w, const P& p, const float (&x)[N]) {
  if (p.full()) {
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
  for (int k = 0; k < K; ++k) v[k] = lm_wave_sum(v[k]);
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

// W waves to a row, PACKS packs a thread; the next row is on its way while one
// is computed.
template <typename E, int W, int PACKS, bool WHOLE>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_norm(NormArgs a) {
  constexpr int N = Pack<E>::N, TEAMS = W == 1 ? 4 : 1;
  typedef Place<N, WHOLE> P;
  __shared__ float lds[2 * W];
  const int tid = W == 1 ? threadIdx.x % 64 : threadIdx.x;
  const int64_t end = lm_offset(a.offsets, a.n, a.T), step = static_cast<int64_t>(gridDim.x) * TEAMS;
  int64_t t = lm_offset(a.offsets, 0, a.T) + static_cast<int64_t>(blockIdx.x) * TEAMS + (W == 1 ? threadIdx.x / 64 : 0);
  const float over_d = 1.f / a.d;
  int turn = 0;
  const auto row = [&](int64_t t, Pack<E>(&x)[PACKS]) {
    const E* p = static_cast<const E*>(a.X) + t * a.ld_X;
#pragma unroll
    for (int i = 0; i < PACKS; ++i) x[i] = load<E>(p, P(tid + i * W * 64, a.d, i == PACKS - 1));
  };
  // the weights stay in registers where they fit
  constexpr bool HELD = PACKS * N <= 32;
  float g[HELD ? PACKS : 1][N], b[HELD ? PACKS : 1][N];
  const auto weights = [&](int i, float(&g)[N], float(&b)[N]) {
    const P p(tid + i * W * 64, a.d, i == PACKS - 1);
    load_f32<N>(a.gamma, p, g);
    if (a.beta) {
      load_f32<N>(a.beta, p, b);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) b[j] = 0.f;
    }
  };
  Pack<E> x[PACKS], next[PACKS];
  if (t < end) row(t, x);
  if constexpr (HELD)
#pragma unroll
    for (int i = 0; i < PACKS; ++i) weights(i, g[i], b[i]);
  for (; t < end; t += step) {
    if (t + step < end) row(t + step, next);
    float sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < PACKS; ++i) {
      const P p(tid + i * W * 64, a.d, i == PACKS - 1);
#pragma unroll
      for (int j = 0; j < N; ++j) sum[0] = WHOLE ? sum[0] + x[i][j] : fmaf(x[i][j], p.own(j), sum[0]);
    }
    row_sum<W, 1>(sum, lds, turn);
    const float mean = sum[0] * over_d;
    float sq[1] = {0.f};
#pragma unroll
    for (int i = 0; i < PACKS; ++i) {
      const P p(tid + i * W * 64, a.d, i == PACKS - 1);
      float part = 0.f;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float c = WHOLE ? x[i][j] - mean : (x[i][j] - mean) * p.own(j);
        part = fmaf(c, c, part);
      }
      sq[0] += p.end ? part : 0.f;
    }
    row_sum<W, 1>(sq, lds, turn);
    const float r = 1.f / sqrtf(fmaf(sq[0], over_d, a.eps));
    E* out = static_cast<E*>(a.out) + t * a.ld_out;
#pragma unroll
    for (int i = 0; i < PACKS; ++i) {
      const P p(tid + i * W * 64, a.d, i == PACKS - 1);
      const int k = HELD ? i : 0;
      if (!HELD) weights(i, g[0], b[0]);
      float y[N];
#pragma unroll
      for (int j = 0; j < N; ++j) y[j] = fmaf((x[i][j] - mean) * r, g[k][j], b[k][j]);
      if (p.end) store<E>(out, p, y);
    }
#pragma unroll
    for (int i = 0; i < PACKS; ++i) x[i] = next[i];
  }
}

// The rows of part number `part` of all rows, a.rows of them, group by group:
// f(group, first, last) for each piece.  Piece and part make a slot of their
// own for the piece's sums, part + group: from one piece to the next, the part
// or the group goes up.
template <typename F>
__device__ __forceinline__ void pieces(const int32_t* offsets, int n, int64_t T, uint32_t rows, uint32_t part, F f) {
  const int lane = threadIdx.x % 64;
  const int64_t o0 = lm_offset(offsets, 0, T), end = lm_offset(offsets, n, T);
  int64_t t = o0 + static_cast<int64_t>(part) * rows;
  const int64_t last = std::min<int64_t>(end, t + rows);
  if (t >= last) return;
  // the last group that starts at t or before, 64 at once
  int i = 0;
  for (int count = n; count > 1;) {
    const int step = (count + 63) / 64, at = lane * step;
    const uint64_t below = __ballot(at < count && lm_offset(offsets, i + at, T) <= t);
    const int k = below ? 63 - __builtin_clzll(below) : 0;
    i += k * step;
    count = std::min(step, count - k * step);
  }
  i = __builtin_amdgcn_readfirstlane(i);
  for (; i < n && t < last; ++i) {
    const int64_t to = std::min(last, lm_offset(offsets, i + 1, T));
    if (to <= t) continue;
    f(i, t, to);
    t = to;
  }
}

template <typename E, int W, int PACKS, bool WHOLE>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_norm_grad(NormArgs a) {
  constexpr int N = Pack<E>::N, TEAMS = W == 1 ? 4 : 1;
  typedef Place<N, WHOLE> P;
  __shared__ float lds[2 * 3 * W];
  const int tid = W == 1 ? threadIdx.x % 64 : threadIdx.x;
  const uint32_t part = blockIdx.x * TEAMS + (W == 1 ? threadIdx.x / 64 : 0);
  if (part >= a.parts_of_rows) return;
  const float over_d = 1.f / a.d;
  float dg[PACKS][N], db[PACKS][N];
  int turn = 0;
  const auto row = [&](int64_t t, Pack<E>(&x)[PACKS], Pack<E>(&dy)[PACKS]) {
    const E* p = static_cast<const E*>(a.X) + t * a.ld_X;
    const E* q = static_cast<const E*>(a.dY) + t * a.ld_dY;
#pragma unroll
    for (int i = 0; i < PACKS; ++i) {
      const P at(tid + i * W * 64, a.d, i == PACKS - 1);
      x[i] = load<E>(p, at);
      dy[i] = load<E>(q, at);
    }
  };
  float g[PACKS][N];
#pragma unroll
  for (int i = 0; i < PACKS; ++i) load_f32<N>(a.gamma, P(tid + i * W * 64, a.d, i == PACKS - 1), g[i]);
  pieces(a.offsets, a.n, a.T, a.rows, part, [&](int group, int64_t first, int64_t last) {
#pragma unroll
    for (int i = 0; i < PACKS; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) dg[i][j] = db[i][j] = 0.f;
    Pack<E> x[PACKS], dy[PACKS], next_x[PACKS], next_dy[PACKS];
    row(first, x, dy);
    for (int64_t t = first; t < last; ++t) {
      if (t + 1 < last) row(t + 1, next_x, next_dy);
      float sum[1] = {0.f};
#pragma unroll
      for (int i = 0; i < PACKS; ++i) {
        const P p(tid + i * W * 64, a.d, i == PACKS - 1);
#pragma unroll
        for (int j = 0; j < N; ++j) sum[0] = WHOLE ? sum[0] + x[i][j] : fmaf(x[i][j], p.own(j), sum[0]);
      }
      row_sum<W, 1>(sum, lds, turn);
      const float mean = sum[0] * over_d;
      // sums of (x - mean)^2, dH and dH (x - mean)
      float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < PACKS; ++i) {
        const P p(tid + i * W * 64, a.d, i == PACKS - 1);
        float part = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float c = WHOLE ? x[i][j] - mean : (x[i][j] - mean) * p.own(j), h = dy[i][j] * g[i][j];
          part = fmaf(c, c, part);
          s[1] = WHOLE ? s[1] + h : fmaf(h, p.own(j), s[1]);
          s[2] = fmaf(h, c, s[2]);
        }
        s[0] += p.end ? part : 0.f;   // (dY is 0 behind the end)
      }
      row_sum<W, 3>(s, lds, turn);
      const float r = 1.f / sqrtf(fmaf(s[0], over_d, a.eps));
      const float m1 = s[1] * over_d, m2 = s[2] * over_d * r;
      E* out = static_cast<E*>(a.out) + t * a.ld_out;
#pragma unroll
      for (int i = 0; i < PACKS; ++i) {
        const P p(tid + i * W * 64, a.d, i == PACKS - 1);
        float y[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float h = (x[i][j] - mean) * r, d = dy[i][j];
          dg[i][j] = fmaf(d, h, dg[i][j]);
          db[i][j] += d;
          y[j] = r * (fmaf(-h, m2, fmaf(d, g[i][j], -m1)));
        }
        if (p.end) store<E>(out, p, y);
      }
#pragma unroll
      for (int i = 0; i < PACKS; ++i) {
        x[i] = next_x[i];
        dy[i] = next_dy[i];
      }
    }
    const int64_t ld = (a.d + 3) / 4 * 4;
    float* sums = a.parts + (part + group) * ld;
#pragma unroll
    for (int i = 0; i < PACKS; ++i) {
      const P p(tid + i * W * 64, a.d, i == PACKS - 1);
      if (p.end == 0) continue;
      store_f32<N>(sums, p, dg[i]);
      if (a.dbeta) store_f32<N>(sums + (static_cast<int64_t>(a.parts_of_rows) + a.n) * ld, p, db[i]);
    }
  });
}

// A thread takes one pack of columns and every 256 / lanes-th row, four of them
// at once.
template <typename E>
__global__ __launch_bounds__(256) void k_linear_grad(LinearGradArgs a, int lanes) {
  constexpr int N = Pack<E>::N;
  __shared__ float lds[256][N + 1];
  const int step = 256 / lanes, tid = threadIdx.x;
  const Place<N> p(static_cast<int>(blockIdx.y) * lanes + tid % lanes, a.C);
  const E* dY = static_cast<const E*>(a.dY);
  const E* Z = static_cast<const E*>(a.Z);
  E* dZ = static_cast<E*>(a.dZ);
  pieces(a.offsets, a.n, a.T, a.rows, blockIdx.x, [&](int group, int64_t first, int64_t last) {
    float sum[N];
#pragma unroll
    for (int j = 0; j < N; ++j) sum[j] = 0.f;
    if (p.end)
      for (int64_t t = first + tid / lanes; t < last; t += 4 * step) {
        Pack<E> dy[4], z[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (t + k * step < last) {
            dy[k] = load<E>(dY + (t + k * step) * a.ld_dY, p);
            if (Z) z[k] = load<E>(Z + (t + k * step) * a.ld_Z, p);
          }
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (t + k * step < last) {
            float y[N];
#pragma unroll
            for (int j = 0; j < N; ++j) y[j] = Z ? dy[k][j] * lm_act_slope(z[k][j], a.act) : dy[k][j];
            if (dZ) store<E>(dZ + (t + k * step) * a.ld_dZ, p, y);
#pragma unroll
            for (int j = 0; j < N; ++j) sum[j] += y[j];
          }
      }
    if (!a.dbias) return;
    for (int s = 128; s >= lanes; s /= 2) {
      if (tid >= s && tid < 2 * s)
#pragma unroll
        for (int j = 0; j < N; ++j) lds[tid][j] = sum[j];
      __syncthreads();
      if (tid < s)
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] += lds[tid + s][j];
    }
    if (tid < lanes && p.end) store_f32<N>(a.parts + (blockIdx.x + group) * ((a.C + 3) / 4 * int64_t{4}), p, sum);
    __syncthreads();
  });
}

// Sums over the pieces of a group: 16 threads for four columns, each takes
// every 16th piece.
struct PieceSum {
  int n, d;
  int64_t T;
  const int32_t* offsets;
  uint32_t rows, slots;
  const float* parts;
  float* out[2];
  int64_t ld_out[2];
};
__global__ __launch_bounds__(256) void k_piece_sum(PieceSum a) {
  __shared__ lm_f32x4 lds[16][17];
  const int which = blockIdx.z, q = threadIdx.x % 16, part = threadIdx.x / 16;
  const int64_t ld = (a.d + 3) / 4 * 4, o0 = lm_offset(a.offsets, 0, a.T);
  for (int i = blockIdx.y; i < a.n; i += gridDim.y) {
    const int64_t first = lm_offset(a.offsets, i, a.T), end = lm_offset(a.offsets, i + 1, a.T);
    uint32_t from = 0, count = 0;
    if (end > first && first >= o0) {
      const uint32_t p0 = static_cast<uint32_t>((first - o0) / a.rows), p1 = static_cast<uint32_t>((end - 1 - o0) / a.rows);
      from = std::min(p0 + i, a.slots);
      count = std::min(p1 - p0 + 1, a.slots - from);
    }
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

int norm_waves(int d) { return d <= 1024 ? 1 : d <= 4096 ? 4 : 16; }

// Rows of a part: about as many parts as run at once, and each with two rows at
// least for every sum that it leaves.  Measured, us with the sums over the
// pieces (8192 x 4096 bf16; 60000 x 1024 bf16; 3001 x 1003 fp32 of 64 groups):
//   512 parts of workgroups, 2048 of waves   63; 110; 26 (4 rows at least)
//   768 and 4096                             62; 97; 23
//   1024 and 4096                            60 (4090 columns 78 for 69); 97; 26 (4 rows)
// Sixteen waves a row (8192 columns and more): 512 parts 71, 768 77.
uint32_t norm_rows(int64_t T, int d) {
  const int w = norm_waves(d);
  return static_cast<uint32_t>(std::max<int64_t>(2, ceil_div(T, w == 1 ? 4096 : w == 4 ? 768 : 512)));
}

int linear_lanes(int packs) {
  int lanes = 64;
  while (lanes > 1 && lanes / 2 >= packs) lanes /= 2;
  return lanes;
}

uint32_t linear_rows(int64_t T, int C) {
  const int64_t tiles = ceil_div(C, 512);
  return static_cast<uint32_t>(std::max<int64_t>(16, ceil_div(T * tiles, 1024)));
}

uint32_t parts_of(int64_t T, uint32_t rows) { return static_cast<uint32_t>(ceil_div(T, rows)); }
uint32_t slots_of(int n, int64_t T, uint32_t rows) { return parts_of(T, rows) + n; }

void launch_piece_sum(const PieceSum& c, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(ceil_div(c.d, 64)), std::min(c.n, 1024), c.out[1] ? 2 : 1);
  k_piece_sum<<<grid, 256, 0, s>>>(c);
}

// The kernels with `packs` packs a thread, of FROM to TO.
template <typename E, int W, int FROM, int TO>
void forward(const NormArgs& a, int packs, hipStream_t s) {
  if constexpr (FROM < TO)
    if (packs > FROM) return forward<E, W, FROM + 1, TO>(a, packs, s);
  constexpr int TEAMS = W == 1 ? 4 : 1, THREADS = W == 1 ? 256 : 64 * W;
  const uint32_t grid = static_cast<uint32_t>(std::min<int64_t>(W == 16 ? 512 : 2048, ceil_div(a.T, TEAMS)));
  if (a.d % Pack<E>::N == 0) k_norm<E, W, FROM, true><<<grid, THREADS, 0, s>>>(a);
  else k_norm<E, W, FROM, false><<<grid, THREADS, 0, s>>>(a);
}
template <typename E, int W, int FROM, int TO>
void backward(const NormArgs& a, int packs, hipStream_t s) {
  if constexpr (FROM < TO)
    if (packs > FROM) return backward<E, W, FROM + 1, TO>(a, packs, s);
  constexpr int TEAMS = W == 1 ? 4 : 1, THREADS = W == 1 ? 256 : 64 * W;
  const uint32_t grid = static_cast<uint32_t>(ceil_div(a.parts_of_rows, TEAMS));
  if (a.d % Pack<E>::N == 0) k_norm_grad<E, W, FROM, true><<<grid, THREADS, 0, s>>>(a);
  else k_norm_grad<E, W, FROM, false><<<grid, THREADS, 0, s>>>(a);
}

template <typename E>
void norm_typed(const NormArgs& a, bool grad, hipStream_t s) {
  constexpr int N = Pack<E>::N;
  if (!grad) {
    // a wave to a row as far as its registers hold one: no barriers
    const int packs = static_cast<int>(ceil_div(a.d, N * 64));
    constexpr int MOST = N == 4 ? 8 : 4;
    if (packs <= MOST) return forward<E, 1, 1, MOST>(a, packs, s);
    if constexpr (N == 4)
      if (packs > 32) return forward<E, 16, 3, 4>(a, (packs + 15) / 16, s);
    return forward<E, 4, N == 4 ? 3 : 2, 8>(a, (packs + 3) / 4, s);
  }
  const int w = norm_waves(a.d), packs = static_cast<int>(ceil_div(a.d, N * 64 * w));
  constexpr int LEAST = N == 4 ? 2 : 1, MOST = N == 4 ? 4 : 2;    // (more than 1024, or 4096, values)
  if (w == 1) return backward<E, 1, 1, MOST>(a, packs, s);
  if (w == 4) return backward<E, 4, LEAST, MOST>(a, packs, s);
  return backward<E, 16, LEAST, MOST>(a, packs, s);
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
  a.parts_of_rows = parts_of(a.T, a.rows);
  if (a.T > 0) norm(a, true, s);
  launch_piece_sum(PieceSum{a.n, a.d, a.T, a.offsets, a.rows, slots_of(a.n, a.T, a.rows), a.parts, {a.dgamma, a.dbeta},
                            {a.ld_dgamma, a.ld_dbeta}}, s);
  return hipGetLastError();
}

int64_t linear_grad_workspace(int n, int64_t T, int C) {
  return int64_t{4} * slots_of(n, T, linear_rows(T, C)) * ((C + 3) / 4 * 4);
}

hipError_t launch_linear_grad(LinearGradArgs a, hipStream_t s) {
  a.rows = linear_rows(a.T, a.C);
  if (a.T > 0) {
    const int packs = static_cast<int>(ceil_div(a.C, a.dtype == DBW_F32 ? 4 : 8));
    const int lanes = linear_lanes(packs);
    const dim3 grid(parts_of(a.T, a.rows), static_cast<uint32_t>(ceil_div(packs, lanes)));
    if (a.dtype == DBW_F32) k_linear_grad<float><<<grid, 256, 0, s>>>(a, lanes);
    else if (a.dtype == DBW_BF16) k_linear_grad<__bf16><<<grid, 256, 0, s>>>(a, lanes);
    else k_linear_grad<_Float16><<<grid, 256, 0, s>>>(a, lanes);
  }
  if (a.dbias)
    launch_piece_sum(PieceSum{a.n, a.C, a.T, a.offsets, a.rows, slots_of(a.n, a.T, a.rows), a.parts, {a.dbias, nullptr}, {a.ld_dbias, 0}}, s);
  return hipGetLastError();
}

}  // namespace dbw
