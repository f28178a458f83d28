// Products of ragged groups on the matrix cores: Y[t] = X[t] W_i,
// dX[t] = dY[t] W_i^T and G_i = sum over the rows of a group of X[t]^T dY[t].
//
// One kernel computes a tile of BM x BN outputs, 64 terms of the sum a step.
// An operand is either contiguous along the sum (X, dY, and W in dX) or along
// the output (W in Y, both operands of G): the first is kept in LDS as rows of
// 64 terms and read 16 bytes a lane, the second as it lies in memory, one row
// a term, and read with the transposing LDS load, so nothing is transposed
// beforehand.  Rows of another group, and what lies behind an edge, are
// replaced by zeros on the way into registers, in both operands: NaN and
// infinities there reach no sum.
//
// Steps are pipelined: the loads of the next one are in flight while the
// present one is multiplied, and go from registers to the other LDS buffer
// after it, with one barrier a step.
//
// v_mfma_f32_16x16x32 takes, in lane l = 16 g + c, row c and terms 8 g .. 8 g
// + 7 of each operand; its result r of a lane is row 4 g + r of the first
// operand, row c of the second.  The output's columns go in as the first
// operand, and tile j of four stands for the columns 16 (c / 4) + 4 j + c % 4
// of 64, so that a lane ends up with 16 consecutive columns of one output row
// and stores 16 bytes at a time.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "dbw_buffer.h"
#include "lm_ops.h"

namespace dbw {
namespace {

constexpr int BK = 64;   // terms of the sum a step

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mma(const lm_u32x4& a, const lm_u32x4& b, f32x4 c, __bf16) {
  typedef __bf16 V __attribute__((ext_vector_type(8)));
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(const lm_u32x4& a, const lm_u32x4& b, f32x4 c, _Float16) {
  typedef _Float16 V __attribute__((ext_vector_type(8)));
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
}

// What a workgroup computes: out[m][n] = sum over k in [k0, k1) of A(m, k) B(n, k)
// for m < rows, n < cols.  A(m, k) is a[m * lda + k], or a[k * lda + m] where
// the operand is contiguous along the output; the same for B.
struct Tile {
  const void* a;
  const void* b;
  void* out;
  int64_t lda, ldb, ldo;
  int64_t k0, k1;
  int rows, cols;
};

// One operand's part of a step: L outputs x BK terms, by THREADS threads.
// SWAP: contiguous along the output.  WIDE: whole 16-byte chunks everywhere.
template <typename E, int L, int THREADS, bool SWAP, bool WIDE>
struct Operand {
  static constexpr int CHUNKS = L * BK / 8 / THREADS;   // 16-byte chunks a thread
  static constexpr int LINE = SWAP ? L / 8 : BK / 8;    // chunks of a line in memory
  static_assert(L * BK / 8 % THREADS == 0 && THREADS % LINE == 0, "whole chunks a thread");
  static constexpr int STEP = THREADS / LINE;           // lines between a thread's chunks
  static constexpr int BYTES = L * BK * 2;

  lm_u32x4 held[CHUNKS];

  // Rows of 64 terms: the chunk of 8 terms is moved by its row, so that the
  // lanes of a fragment (rows 4 a + b of tiles, see below) meet in no bank.
  static __device__ __forceinline__ int turn(int row) { return (row & 3) | (((row >> 2) ^ (row >> 4)) & 1) << 2; }

  __device__ __forceinline__ void load(const E* p, int64_t ld, int64_t k, int64_t k1, int length, int tid) {
    const int line = tid / LINE, chunk = tid % LINE;
    const E* base = SWAP ? p + k * ld : p + k;
    const int64_t left = k1 - k;                         // terms from k on
    if (WIDE) {
      const __amdgpu_buffer_rsrc_t r = make_rsrc(base, static_cast<uint32_t>(kMaxBufferBytes));
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        const int at = line + i * STEP;
        const bool in = SWAP ? at < left && chunk * 8 < length : at < length && chunk * 8 < left;
        const uint32_t off = in ? static_cast<uint32_t>((at * ld + chunk * 8) * 2) : kOutOfRange;
        held[i] = __builtin_bit_cast(lm_u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
      }
    } else {
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        const int at = line + i * STEP;
        const int64_t lines = SWAP ? left : length, in_line = (SWAP ? length : left) - chunk * 8;
        lm_u32x4 v = {0, 0, 0, 0};
        if (at < lines && in_line > 0) {
          const E* q = base + at * ld + chunk * 8;
          if (in_line >= 8) {
            v = *reinterpret_cast<const lm_u32x4_any*>(q);
          } else {
            typedef E V __attribute__((ext_vector_type(8)));
            V x = __builtin_bit_cast(V, v);
#pragma unroll
            for (int j = 0; j < 7; ++j)
              if (j < in_line) x[j] = q[j];
            v = __builtin_bit_cast(lm_u32x4, x);
          }
        }
        held[i] = v;
      }
    }
  }

  __device__ __forceinline__ void store(char* lds, int tid) const {
    const int line = tid / LINE, chunk = tid % LINE;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int at = line + i * STEP;
      if (SWAP) {
        // pieces of four columns, piece ^ (at & 3), and 32 columns apart every
        // other eight lines: the lines 8 g + r that the transposing load
        // takes at once meet in no bank
        const int c = chunk ^ ((at >> 1) & 1) ^ (L >= 128 ? ((at >> 3) & 1) << 3 : 0);
        const lm_u32x4 v = held[i];
        const lm_u32x4 w = {v[2], v[3], v[0], v[1]};
        *reinterpret_cast<lm_u32x4*>(lds + at * (L * 2) + c * 16) = at & 1 ? w : v;
      } else {
        *reinterpret_cast<lm_u32x4*>(lds + at * (BK * 2) + (chunk ^ turn(at)) * 16) = held[i];
      }
    }
  }

  // Fragment of a lane: terms 32 kk + 8 g .. + 7 of output `first` + (row c
  // of tile j).  PERM: tile j of each 64 outputs takes 16 (c / 4) + 4 j + c % 4.
  template <bool PERM>
  static __device__ __forceinline__ lm_u32x4 fragment(const char* lds, int first, int tile, int kk, int lane) {
    const int c = lane % 16, g = lane / 16;
    const int base = PERM ? first + tile / 4 * 64 : first + tile * 16, j = tile % 4;
    if (SWAP) {
      const int r = c / 4, at = kk * 32 + g * 8 + r;     // and at + 4: the same low bits
      const int piece = PERM ? base / 4 + 4 * (c % 4) + j : base / 4 + c % 4;
      const int p = (piece ^ r) ^ (L >= 128 ? (g & 1) << 4 : 0);
      const char* q = lds + at * (L * 2) + p * 8;
      typedef __attribute__((address_space(3))) s16x4* P;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(q));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(q + 4 * L * 2));
      const lm_u32x2 x = __builtin_bit_cast(lm_u32x2, lo), y = __builtin_bit_cast(lm_u32x2, hi);
      return lm_u32x4{x[0], x[1], y[0], y[1]};
    }
    const int row = PERM ? base + 16 * (c / 4) + 4 * j + c % 4 : base + c;
    return *reinterpret_cast<const lm_u32x4*>(lds + row * (BK * 2) + ((kk * 4 + g) ^ turn(row)) * 16);
  }
};

// 16 consecutive outputs of one row, `left` of them inside.
template <typename E>
__device__ __forceinline__ void store16(E* p, const float (&x)[16], int left) {
  constexpr int N = 16 / sizeof(E);
  typedef E V __attribute__((ext_vector_type(16 / sizeof(E))));
#pragma unroll
  for (int q = 0; q < 16 / N; ++q) {
    V v;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = static_cast<E>(x[q * N + j]);
    if (left >= (q + 1) * N) {
      *reinterpret_cast<lm_u32x4_any*>(p + q * N) = __builtin_bit_cast(lm_u32x4, v);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (q * N + j < left) p[q * N + j] = v[j];
    }
  }
}

template <typename E, int BM, int BN, int WM, int WN, bool A_SWAP, bool B_SWAP, bool WIDE>
__device__ __forceinline__ void product(const Tile& t, bool out_f32, char* lds) {
  constexpr int THREADS = (BM / WM) * (BN / WN) * 64;
  constexpr int TM = WM / 16, TN = WN / 16;
  constexpr bool PERM = WM % 64 == 0;
  static_assert(WN % 64 == 0, "a lane's columns are those of four tiles");
  typedef Operand<E, BM, THREADS, A_SWAP, WIDE> OpA;
  typedef Operand<E, BN, THREADS, B_SWAP, WIDE> OpB;
  constexpr int STAGE = OpA::BYTES + OpB::BYTES;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int m0 = wave / (BN / WN) * WM, n0 = wave % (BN / WN) * WN;
  const E* a = static_cast<const E*>(t.a);
  const E* b = static_cast<const E*>(t.b);

  f32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  OpA A;
  OpB B;
  int cur = 0;
  if (t.k0 < t.k1) {
    A.load(a, t.lda, t.k0, t.k1, t.rows, tid);
    B.load(b, t.ldb, t.k0, t.k1, t.cols, tid);
    A.store(lds, tid);
    B.store(lds + OpA::BYTES, tid);
  }
  __syncthreads();
  for (int64_t k = t.k0; k < t.k1; k += BK) {
    const bool more = k + BK < t.k1;
    if (more) {
      A.load(a, t.lda, k + BK, t.k1, t.rows, tid);
      B.load(b, t.ldb, k + BK, t.k1, t.cols, tid);
    }
    const char* la = lds + cur * STAGE;
    const char* lb = la + OpA::BYTES;
#pragma unroll
    for (int kk = 0; kk < BK / 32; ++kk) {
      lm_u32x4 fb[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[j] = OpB::template fragment<true>(lb, n0, j, kk, lane);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const lm_u32x4 fa = OpA::template fragment<PERM>(la, m0, i, kk, lane);
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mma(fb[j], fa, acc[i][j], E{});
      }
    }
    if (more) {
      cur ^= 1;
      A.store(lds + cur * STAGE, tid);
      B.store(lds + cur * STAGE + OpA::BYTES, tid);
      __syncthreads();
    }
  }

  const int c = lane % 16, g = lane / 16;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int m = m0 + (PERM ? i / 4 * 64 + 16 * (c / 4) + 4 * (i % 4) + c % 4 : i * 16 + c);
    if (m >= t.rows) continue;
#pragma unroll
    for (int q = 0; q < TN / 4; ++q) {
      const int n = n0 + q * 64 + 16 * g;
      if (n >= t.cols) continue;
      float x[16];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[4 * j + r] = acc[i][4 * q + j][r];
      const int64_t at = static_cast<int64_t>(m) * t.ldo + n;
      if (out_f32)
        store16(static_cast<float*>(t.out) + at, x, t.cols - n);
      else
        store16(static_cast<E*>(t.out) + at, x, t.cols - n);
    }
  }
}

struct GroupArgs {
  const int32_t* offsets;
  const void* a;
  const void* b;
  void* out;         // or the partial outputs, float [splits][part]
  int form, n, d, C;
  int64_t T, ld_d, ld_C, ld_W, st_W;
  int splits;
  int64_t part;
  uint32_t row_tiles, col_tiles, blocks;
  int out_f32, out_bytes;
};

// Terms of one part of a sum of `length` terms: whole steps.
__device__ __forceinline__ int64_t split_of(int64_t length, int splits) {
  return ((length + BK - 1) / BK + splits - 1) / splits * BK;
}

template <typename E, int BM, int BN, int WM, int WN, int FORM, bool WIDE>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64, 2) void k_group(GroupArgs g) {
  constexpr bool A_SWAP = FORM == DBW_GROUP_WEIGHT_GRAD, B_SWAP = FORM != DBW_GROUP_INPUT_GRAD;
  __shared__ __align__(16) char lds[2 * (BM + BN) * BK * 2];
  // Workgroups go to the eight XCDs in turn; consecutive tiles share an
  // operand, so each XCD (and its L2) takes a run of them.
  const uint32_t per = (g.blocks + 7) / 8;
  const uint32_t id = blockIdx.x % 8 * per + blockIdx.x / 8;
  if (id >= g.blocks) return;
  const int lane = threadIdx.x % 64;
  Tile t;
  if (FORM == DBW_GROUP_WEIGHT_GRAD) {
    uint32_t q = id;
    const uint32_t rt = q % g.row_tiles;
    q /= g.row_tiles;
    const uint32_t ct = q % g.col_tiles;
    q /= g.col_tiles;
    const int split = q % g.splits;
    const int group = q / g.splits;
    const int64_t first = lm_offset(g.offsets, group, g.T), end = lm_offset(g.offsets, group + 1, g.T);
    const int64_t length = end > first ? end - first : 0;
    const int64_t step = split_of(length, g.splits);
    const int m = rt * BM, n = ct * BN;
    t.a = static_cast<const E*>(g.a) + m;
    t.b = static_cast<const E*>(g.b) + n;
    t.lda = g.ld_d;
    t.ldb = g.ld_C;
    t.k0 = first + std::min<int64_t>(length, split * step);
    t.k1 = first + std::min<int64_t>(length, (split + 1) * step);
    t.rows = std::min(BM, g.d - m);
    t.cols = std::min(BN, g.C - n);
    if (g.splits > 1) {
      t.ldo = g.C;
      t.out = static_cast<float*>(g.out) + split * g.part + (static_cast<int64_t>(group) * g.d + m) * g.C + n;
    } else {
      t.ldo = g.ld_W;
      t.out = static_cast<char*>(g.out) + (group * g.st_W + m * g.ld_W + n) * g.out_bytes;
    }
  } else {
    const int K = FORM == DBW_GROUP_FORWARD ? g.d : g.C, N = FORM == DBW_GROUP_FORWARD ? g.C : g.d;
    uint32_t q = id;
    const int split = q % g.splits;
    q /= g.splits;
    // bands of eight row tiles, rows fastest: workgroups that run together
    // share rows and columns
    const uint32_t band = q / (8 * g.col_tiles), in_band = q % (8 * g.col_tiles);
    const uint32_t height = std::min(8u, g.row_tiles - band * 8);
    const uint32_t rt = band * 8 + in_band % height, ct = in_band / height;
    if (rt >= g.row_tiles) return;
    // the group of row tile rt: sums of the groups' tiles, 64 groups at once
    // (T < 2^31; lane values go to scalars, which keeps the addresses scalar)
    int group = -1, first = 0, end = 0, tile = 0;
    if (g.st_W == 0) {
      first = static_cast<int>(lm_offset(g.offsets, 0, g.T));
      end = static_cast<int>(lm_offset(g.offsets, g.n, g.T));
      tile = rt;
      group = 0;
    } else {
      uint32_t before = 0;   // tiles of the groups passed
      for (int i0 = 0; i0 < g.n; i0 += 64) {
        const int i = i0 + lane;
        int o = 0, e = 0;
        if (i < g.n) {
          o = static_cast<int>(lm_offset(g.offsets, i, g.T));
          e = static_cast<int>(lm_offset(g.offsets, i + 1, g.T));
        }
        const uint32_t tiles = e > o ? (static_cast<uint32_t>(e - o) + BM - 1) / BM : 0;
        const uint32_t sum = before + lm_wave_scan(tiles, lane);
        const uint64_t past = __ballot(sum > rt);
        if (past) {
          const int l = __builtin_ctzll(past);
          group = i0 + l;
          first = __builtin_amdgcn_readlane(o, l);
          end = __builtin_amdgcn_readlane(e, l);
          tile = rt - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(tiles, l));
          break;
        }
        before = __builtin_amdgcn_readlane(sum, 63);
      }
    }
    const int64_t row = first + static_cast<int64_t>(tile) * BM;
    if (group < 0 || row >= end) return;
    const int n = ct * BN;
    const int64_t step = split_of(K, g.splits);
    t.lda = FORM == DBW_GROUP_FORWARD ? g.ld_d : g.ld_C;
    t.ldb = g.ld_W;
    t.a = static_cast<const E*>(g.a) + row * t.lda;
    t.b = static_cast<const E*>(g.b) + group * g.st_W + (FORM == DBW_GROUP_FORWARD ? n : n * g.ld_W);
    t.k0 = std::min<int64_t>(K, split * step);
    t.k1 = std::min<int64_t>(K, (split + 1) * step);
    t.rows = static_cast<int>(std::min<int64_t>(BM, end - row));
    t.cols = std::min(BN, N - n);
    if (g.splits > 1) {
      t.ldo = N;
      t.out = static_cast<float*>(g.out) + split * g.part + row * N + n;
    } else {
      t.ldo = FORM == DBW_GROUP_FORWARD ? g.ld_C : g.ld_d;
      t.out = static_cast<char*>(g.out) + (row * t.ldo + n) * g.out_bytes;
    }
  }
  product<E, BM, BN, WM, WN, A_SWAP, B_SWAP, WIDE>(t, g.splits > 1 || g.out_f32, lds);
}

// out = the sum of the partial outputs, in the order of the parts.
template <typename O>
__global__ __launch_bounds__(256) void k_group_sum(GroupArgs g, const float* __restrict__ parts) {
  const bool grad = g.form == DBW_GROUP_WEIGHT_GRAD;
  const int N = g.form == DBW_GROUP_INPUT_GRAD ? g.d : g.C;
  // rows outside the groups stay as they were
  const int64_t first = grad ? 0 : lm_offset(g.offsets, 0, g.T);
  const int64_t end = grad ? static_cast<int64_t>(g.n) * g.d : lm_offset(g.offsets, g.n, g.T);
  const int64_t all = (end - first) * N;
  for (int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4; i < all;
       i += static_cast<int64_t>(gridDim.x) * 1024) {
    const float* p = parts + first * N + i;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (i + 4 <= all) {
      for (int s = 0; s < g.splits; ++s) {
        const lm_f32x4 v = *reinterpret_cast<const lm_f32x4_any*>(p + s * g.part);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] += v[j];
      }
    } else {
      for (int s = 0; s < g.splits; ++s)
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (i + j < all) x[j] += p[s * g.part + j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i + j >= all) break;
      const int64_t row = first + (i + j) / N, n = (i + j) % N;
      const int64_t at = grad ? row / g.d * g.st_W + row % g.d * g.ld_W + n
                              : row * (g.form == DBW_GROUP_FORWARD ? g.ld_C : g.ld_d) + n;
      static_cast<O*>(g.out)[at] = static_cast<O>(x[j]);
    }
  }
}

enum GroupVariant { SMALL = 0, MIDDLE = 1, LARGE = 2 };
struct VariantSize {
  int bm, bn;
};
constexpr VariantSize kSize[] = {{32, 256}, {128, 128}, {256, 256}};

template <typename E, int FORM, bool WIDE>
void launch_variant(const GroupPlan& plan, const GroupArgs& g, uint32_t grid, hipStream_t s) {
  if (plan.variant == LARGE)
    k_group<E, 256, 256, 128, 64, FORM, WIDE><<<grid, 512, 0, s>>>(g);
  else if (plan.variant == MIDDLE || FORM == DBW_GROUP_WEIGHT_GRAD)
    k_group<E, 128, 128, 64, 64, FORM, WIDE><<<grid, 256, 0, s>>>(g);
  else if constexpr (FORM != DBW_GROUP_WEIGHT_GRAD)
    k_group<E, 32, 256, 32, 64, FORM, WIDE><<<grid, 256, 0, s>>>(g);
}
template <typename E, int FORM>
void launch_wide(bool wide, const GroupPlan& plan, const GroupArgs& g, uint32_t grid, hipStream_t s) {
  if (wide)
    launch_variant<E, FORM, true>(plan, g, grid, s);
  else
    launch_variant<E, FORM, false>(plan, g, grid, s);
}
template <typename E>
void launch_form(bool wide, const GroupPlan& plan, const GroupArgs& g, uint32_t grid, hipStream_t s) {
  if (g.form == DBW_GROUP_FORWARD)
    launch_wide<E, DBW_GROUP_FORWARD>(wide, plan, g, grid, s);
  else if (g.form == DBW_GROUP_INPUT_GRAD)
    launch_wide<E, DBW_GROUP_INPUT_GRAD>(wide, plan, g, grid, s);
  else
    launch_wide<E, DBW_GROUP_WEIGHT_GRAD>(wide, plan, g, grid, s);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

GroupPlan group_plan(const dbw_group_shape& p) {
  GroupPlan plan;
  const bool grad = p.form == DBW_GROUP_WEIGHT_GRAD;
  const int64_t groups = p.st_W == 0 && !grad ? 1 : p.n;
  const int64_t M = grad ? p.d : p.T, N = p.form == DBW_GROUP_INPUT_GRAD ? p.d : p.C;
  const int64_t rows = grad ? M : std::max<int64_t>(1, p.T / groups);   // of one group, on average
  const auto tiles = [&](int v) {
    const int64_t per = ceil_div(rows, kSize[v].bm) * ceil_div(N, kSize[v].bn);
    return per * groups;
  };
  plan.variant = rows <= 48 && !grad ? SMALL : tiles(LARGE) >= 512 && rows >= 512 ? LARGE : MIDDLE;
  const VariantSize size = kSize[plan.variant];
  // every group may end in a tile of its own
  plan.row_tiles = grad ? ceil_div(p.d, size.bm)
                        : std::min<int64_t>(p.T, p.T / size.bm + std::min<int64_t>(groups, p.T));
  plan.col_tiles = ceil_div(N, size.bn);
  const int64_t K = grad ? p.T / p.n : p.form == DBW_GROUP_FORWARD ? p.d : p.C;
  const int64_t blocks = std::max<int64_t>(1, tiles(plan.variant));
  plan.splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({512 / blocks, K / 256, 64})));
  plan.part = grad ? static_cast<int64_t>(p.n) * p.d * p.C : p.T * N;
  plan.blocks = plan.row_tiles * plan.col_tiles * plan.splits * (grad ? p.n : 1);
  return plan;
}

hipError_t launch_group(const dbw_group_shape& p, const GroupPlan& plan, const int32_t* offsets, const void* a,
                        const void* b, void* out, float* workspace, hipStream_t s) {
  const bool grad = p.form == DBW_GROUP_WEIGHT_GRAD;
  if (!grad && p.T == 0) return hipSuccess;
  GroupArgs g{};
  g.offsets = offsets; g.a = a; g.b = b; g.form = p.form; g.n = p.n; g.d = p.d; g.C = p.C;
  g.T = p.T; g.ld_d = p.ld_d; g.ld_C = p.ld_C; g.ld_W = p.ld_W;
  g.st_W = grad && p.n == 1 ? 0 : p.st_W;
  g.splits = plan.splits; g.part = plan.part;
  g.row_tiles = static_cast<uint32_t>(plan.row_tiles);
  g.col_tiles = static_cast<uint32_t>(plan.col_tiles);
  g.out_f32 = p.out_dtype == DBW_F32;
  g.out_bytes = elem_bytes(p.out_dtype);
  g.blocks = static_cast<uint32_t>(plan.blocks);
  g.out = plan.splits > 1 ? workspace : out;
  // whole chunks of 16 bytes: every row starts at one and ends with one
  const auto even = [](const void* q, int64_t ld) { return reinterpret_cast<uintptr_t>(q) % 16 == 0 && ld % 8 == 0; };
  bool wide = p.d % 8 == 0 && p.C % 8 == 0;
  if (p.form == DBW_GROUP_FORWARD)
    wide = wide && even(a, p.ld_d) && even(b, p.ld_W) && p.st_W % 8 == 0;
  else if (p.form == DBW_GROUP_INPUT_GRAD)
    wide = wide && even(a, p.ld_C) && even(b, p.ld_W) && p.st_W % 8 == 0;
  else
    wide = wide && even(a, p.ld_d) && even(b, p.ld_C);
  const uint32_t grid = (g.blocks + 7) / 8 * 8;
  if (p.dtype == DBW_BF16)
    launch_form<__bf16>(wide, plan, g, grid, s);
  else
    launch_form<_Float16>(wide, plan, g, grid, s);
  if (plan.splits > 1) {
    g.out = out;
    const uint32_t sums = static_cast<uint32_t>(std::max<int64_t>(1, std::min<int64_t>(ceil_div(plan.part, 1024), 2048)));
    if (p.out_dtype == DBW_F32)
      k_group_sum<float><<<sums, 256, 0, s>>>(g, workspace);
    else if (p.dtype == DBW_BF16)
      k_group_sum<__bf16><<<sums, 256, 0, s>>>(g, workspace);
    else
      k_group_sum<_Float16><<<sums, 256, 0, s>>>(g, workspace);
  }
  return hipGetLastError();
}

}  // namespace dbw
