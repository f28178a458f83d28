// Causal attention over packed sequences, and its gradients.
//   k_attention       O and lse: a workgroup takes 128 queries of a head
//   k_attention_dq    dQ, and delta = dO . O of each query: the same
//   k_attention_dkv   dK and dV: a workgroup takes 64 keys of a head of keys
//   k_attention_join  dK and dV where several share them
//
// v_mfma_f32_32x32x16 takes, in lane l = 32 h + c, row c and terms 8 h .. 8 h +
// 7 of each operand; its result r of a lane is row 8 (r / 4) + 4 h + r % 4 of
// the first operand, row c of the second.  A wave takes 32 queries as the
// second operand of S^T = K Q^T, so that a lane has 16 keys of one query: the
// softmax needs one exchange between the halves of a wave.  Its exponentials,
// packed as they are, are terms 4 h .. 4 h + 3 and 8 + 4 h .. of sixteen keys;
// the order of terms does not matter, so they are the second operand of O^T =
// V^T P^T without any exchange, when V's transposing loads take the same keys.
// The gradients do the same with K^T, and, with keys for queries, with Q^T and
// dO^T.
//
// A pass over the keys keeps the running maximum and sum of a query; sums are
// scaled only when a maximum has grown by 2^8 (a wave then spends 64 products on
// it; on random rows, in the first stages alone).  The gradients form S and dO V^T
// once for dQ and once for dK and dV, seven products for five: dK and dV, and dQ,
// are then sums of one workgroup in a fixed order, without atomics or arrays of T x T
// (a workgroup for keys that adds to dQ would need fp32 atomics whose order is
// not fixed).
//
// What bounds it.  The next stage's way to LDS, in every step: the compiler cannot
// tell the stage that transposing reads take from the one that loads are filling,
// and waits for all loads before the first of these reads, so that a load overlaps
// the first products and the exponentials of its step only.  (As statements with
// their own wait these reads were slower: forward 64 us for 62,
// dK and dV 142 for 129 in the ragged batch below.)  Long
// sequences besides: the matrix cores at the clock they hold under load; 1 sequence of
// 16384 tokens, 8 heads on 2 of 128, forward 529 to 560 us from box to box, 980 to 1040
// TFLOP/s (a library product 1250), 632 in a run of calls; vector work, 150 instructions and
// 32 exponentials for 32 products, runs beside the products of the other wave of a
// SIMD only in part (cores busy 60% of the cycles).  Ragged batches: the tiles on the diagonal,
// start and end of each workgroup, and the last of them; 8 sequences, 8192 tokens, 16
// heads on 4 of 128: 61, 88 and 133 us in bf16, 670, 690 and 610 TFLOP/s, cores busy 33 to
// 38%; 62, 91 and 143 in fp16.  Short sequences: the chain from offsets to keys to products, some
// 5 us a workgroup (50 sequences, 5000 tokens, 12 heads of 80, fp16: 15, 28 and 28
// us).  LDS is read without conflicts (with lines turned for 32 banks half of its cycles
// were).  Tried, no gain: the priority of waves raised for products.  Not tried: softmax
// of one stage beside the products of the next within a wave, for which 256
// registers do not hold 128 values a head.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "dbw_buffer.h"
#include "lm_ops.h"
#include "lm_tiles.h"

namespace dbw {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mma(const lm_u32x4& a, const lm_u32x4& b, const f32x16& c, __bf16) {
  typedef __bf16 V __attribute__((ext_vector_type(8)));
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(const lm_u32x4& a, const lm_u32x4& b, const f32x16& c, _Float16) {
  typedef _Float16 V __attribute__((ext_vector_type(8)));
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 zero16() {
  return f32x16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
}

// The halves of a wave exchange: a's upper and b's lower one.  (The waits are
// those between a vector result and this instruction.)
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {
  asm volatile("s_nop 3\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
}
__device__ __forceinline__ float max_halves(float x) {
  uint32_t a = __builtin_bit_cast(uint32_t, x), b = a;
  swap_halves(a, b);
  return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
__device__ __forceinline__ float sum_halves(float x) {
  uint32_t a = __builtin_bit_cast(uint32_t, x), b = a;
  swap_halves(a, b);
  return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}

// Rows of DP values in LDS, as a stage of ROWS of them.  A line's chunks of 16
// bytes are turned by its number, so that the lanes that read at once meet in
// none of the 64 banks: sixteen that read a chunk of sixteen lines, or 32 that
// read 64 bytes of four lines by the transposing load.
template <int DP, int ROWS, int THREADS>
struct Rows {
  static constexpr int LINE = DP / 8;                     // chunks of a line
  static constexpr int CHUNKS = ROWS * LINE / THREADS;    // a thread
  static constexpr int BYTES = ROWS * DP * 2;
  // With 128 values, a thread's chunks lie whole periods of turn() apart: one offset
  // does, with a scalar one.  With it, and with line(), dK and dV's loop has no
  // scratch, whose loads wait for the next stage (8 sequences, 8192 tokens, 16 heads on 4:
  // 145 -> 143 us in bf16, 172 -> 142 in fp16).  With 64 values registers suffice, and the
  // scalar ones would not.
  static constexpr bool EVEN = DP == 128 && THREADS / LINE % 16 == 0;
  static constexpr int OFFSETS = EVEN ? 1 : CHUNKS;
  static_assert(DP == 64 || DP == 96 || DP == 128, "turn() is for these");
  static_assert(ROWS * LINE % THREADS == 0, "whole chunks a thread");
  static __device__ __forceinline__ int turn(int line) {
    const int low = line >> 2 & 3;
    return DP == 128 ? (line & 3) << 2 | low : DP == 64 ? (line >> 1 & 1) << 2 | low : low;
  }
  // Byte offset of thread tid's chunk i from the stage's first row, or one
  // behind every buffer (such loads give 0): of `left` rows, of D values each.
  static __device__ __forceinline__ uint32_t offset(int64_t token, int left, int D, int tid, int i) {
    const int id = i * THREADS + tid, line = id / LINE, chunk = id % LINE ^ turn(line);
    return line < left && chunk * 8 < D ? static_cast<uint32_t>(line * token * 2 + chunk * 16) : kOutOfRange;
  }
  static __device__ __forceinline__ void load(const char* p, int64_t token, int left, int D, char* lds, int wave,
                                              int lane, const uint32_t (&off)[OFFSETS]) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(p, static_cast<uint32_t>(kMaxBufferBytes));
    if (left >= ROWS) {
      const uint32_t step = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(token) * (THREADS / LINE * 2));
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i)
        load_lds(r, lds + (i * (THREADS / 64) + wave) * 1024, off[EVEN ? 0 : i], EVEN ? i * step : 0);
    } else {
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i)
        load_lds(r, lds + (i * (THREADS / 64) + wave) * 1024, offset(token, left, D, wave * 64 + lane, i));
    }
  }
  // Terms 16 kk + 8 h .. + 7 of line first + c (first: a multiple of 32).
  static __device__ __forceinline__ lm_u32x4 row(const char* lds, int first, int kk, int lane) {
    const int c = lane % 32, h = lane / 32;
    return *reinterpret_cast<const lm_u32x4*>(lds + (first + c) * (DP * 2) + ((2 * kk + h) ^ turn(c)) * 16);
  }
  // The same from the address of a lane's chunk 0, where lines are 256 bytes from a
  // multiple of that on: chunks' numbers join by exclusive or, and one register
  // holds what would be eight.
  static __device__ __forceinline__ uint32_t line(const char* lds, int first, int lane) {
    const int c = lane % 32, h = lane / 32;
    typedef __attribute__((address_space(3))) const char* P;
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((P)(lds + (first + c) * (DP * 2) + (h ^ turn(c)) * 16)));
  }
  static __device__ __forceinline__ lm_u32x4 row(uint32_t line, int kk) {
    static_assert(DP == 128, "an exclusive or stays in the line");
    typedef __attribute__((address_space(3))) const lm_u32x4* P;
    return *(P)(line ^ kk * 32);
  }
  // Addresses of a lane for column(): of the columns 32 i + 16 (lane / 16 % 2)
  // + 4 q .. + 3 of line 4 h + r, with r and q from lane % 16 = 4 r + q.
  static __device__ __forceinline__ void columns(const char* lds, int lane, uint32_t (&p)[DP / 32]) {
    const int q = lane % 4, line = lane / 32 * 4 + lane % 16 / 4;
    typedef __attribute__((address_space(3))) const char* P;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
      p[i] = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(
          (P)(lds + line * (DP * 2) + ((4 * i + lane / 16 % 2 * 2 + q / 2) ^ turn(line)) * 16 + q % 2 * 8)));
  }
  // Sixteen lines from AT bytes behind them on, transposed: in lane 32 h + c,
  // column 32 i + c of lines 4 h .. + 3 and 8 + 4 h .. + 3 (eight lines on, the
  // turn differs by two chunks).  The reads are builtins, whose waits the compiler
  // places: for their results, and, before the first of a step, for every load on
  // its way to LDS.
  template <int AT, int N>
  static __device__ __forceinline__ void column(const uint32_t (&p)[N], lm_u32x4 (&f)[N]) {
    typedef short S4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) S4* P;
    lm_u32x2 x[N][2];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i][0] = __builtin_bit_cast(lm_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p[i] + AT)));
      x[i][1] = __builtin_bit_cast(lm_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)((p[i] ^ 32) + AT + 8 * DP * 2)));
    }
    join(x, f);
  }
  template <int N>
  static __device__ __forceinline__ void join(const lm_u32x2 (&x)[N][2], lm_u32x4 (&f)[N]) {
    static_assert(ROWS * DP * 2 <= 65536, "offsets have sixteen bits");
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = lm_u32x4{x[i][0][0], x[i][0][1], x[i][1][0], x[i][1][1]};
  }
};

// Address of row `row` of a head's rows.
__device__ __forceinline__ char* at(const HeadRows& r, int64_t row, int head) {
  return r.p + (row * r.token + head * r.head) * 2;
}

// Rows first + c of a head as a wave's operand in registers; rows from `left`
// on are 0.
template <int DP>
__device__ __forceinline__ void operand(const char* first, int64_t token, int left, int D, int lane,
                                        lm_u32x4 (&f)[DP / 16]) {
  const __amdgpu_buffer_rsrc_t r = make_rsrc(first, static_cast<uint32_t>(kMaxBufferBytes));
  const int c = lane % 32, h = lane / 32;
#pragma unroll
  for (int kk = 0; kk < DP / 16; ++kk) {
    const uint32_t off =
        c < left && 16 * kk + 8 * h < D ? static_cast<uint32_t>((c * token + 16 * kk + 8 * h) * 2) : kOutOfRange;
    f[kk] = __builtin_bit_cast(lm_u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
  }
}

// A wave's results, transposed: column c of tile i is row first + c, of which
// a lane has values 32 i + 8 (r / 4) + 4 h + r % 4; times `by`.
template <typename E, int DP>
__device__ __forceinline__ void write_rows(char* first, int64_t token, int left, int D, int lane,
                                           const f32x16 (&x)[DP / 32], float by) {
  const int c = lane % 32, h = lane / 32;
#pragma unroll
  for (int i = 0; i < DP / 32; ++i)
#pragma unroll
    for (int k = 0; k < 16; k += 8) {
      // the halves exchange, so that each has eight values in a row
      uint32_t a0 = pack2<E>(x[i][k] * by, x[i][k + 1] * by), a1 = pack2<E>(x[i][k + 2] * by, x[i][k + 3] * by);
      uint32_t b0 = pack2<E>(x[i][k + 4] * by, x[i][k + 5] * by), b1 = pack2<E>(x[i][k + 6] * by, x[i][k + 7] * by);
      swap_halves(a0, b0);
      swap_halves(a1, b1);
      const int d = 32 * i + 2 * k + 8 * h;
      if (c < left && d < D) *reinterpret_cast<lm_u32x4*>(first + (c * token + d) * 2) = lm_u32x4{a0, a1, b0, b1};
    }
}

// Results r = 8 u .. 8 u + 7 of a lane, as eight terms of an operand.
template <typename E>
__device__ __forceinline__ lm_u32x4 terms(const f32x16& x, int u) {
  return lm_u32x4{pack2<E>(x[8 * u], x[8 * u + 1]), pack2<E>(x[8 * u + 2], x[8 * u + 3]),
                  pack2<E>(x[8 * u + 4], x[8 * u + 5]), pack2<E>(x[8 * u + 6], x[8 * u + 7])};
}

__device__ __forceinline__ int place(int r, int h) { return 8 * (r / 4) + 4 * h + r % 4; }

constexpr int BM = 128, BN = 64;       // queries of a workgroup, keys of a stage
constexpr int KEYS = kAttentionKeys;   // for dK and dV: keys of a workgroup
// Workgroups below which eight waves work on a tile rather than four.  Forward,
// dQ, and dK with dV, us with four and eight waves: 1 sequence of 8192 tokens, 4
// heads of 64 (260 and 516 workgroups) 110, 159, 137 and 84, 108, 104; 1 of 8192, 8
// heads of 128 (520) 194, 284 and 154, 212; 16 of 256 tokens, 8 heads of 64 (384 and
// 640) 12.0, 15.6, 13.7 and 11.6, 16.6, 25: short sequences' keys see too few
// queries for more than four waves.
constexpr int64_t kFewTiles = 640;
// Largest size of a maximum, as an exponent of 2, up to which exponents are
// formed as S scale log2(e) - x with a rounded x = m scale log2(e), in one
// instruction: x is off by 2^-15 then.  Beyond, that would tell: 2^-4 at 2^21,
// where a row's terms have different x; above 2^28 fp16 cannot hold P, and above
// 2^31 exponentials are infinite or all 0.  A wave with such a row subtracts
// before it scales, (S - m) scale log2(e), in one instruction more.  The times of
// ordinary rows are the same with and without (16384 tokens 541 us).  The
// gradients have lse alone, and dQ's kernel forms maximum and sum again for 128
// queries of which one is beyond; all others pay up to 2% of the
// gradients' time for the choice.
constexpr float kFar = 1024.f;
constexpr float kLn2 = 0.693147180559945309f;

// What a workgroup works on: rows first .. of a sequence [start, end) and a head.
struct Work {
  LmChunk rows;
  int head;
};

// Tile number `rank` of all sequences' tiles of `rows` rows, those with the most
// keys (LAST: the last tiles of long sequences) or queries (the first ones) to
// pass first: workgroups start in the order of their numbers, and with the
// longest at the end the others would wait for them (8 sequences of 8192 tokens,
// 16 heads on 4 of 128: 72, 107 and 173 us for the three kernels with tiles in
// the sequences' order, 64, 95 and 142 with this one and LDS free of conflicts).  With w the tiles to pass, its
// own included, the tiles with w or more are sum_i max(0, tiles_i - w + 1).
// kSorted sequences at most: beyond, chunks in the sequences' order.
constexpr int kSorted = 256;
template <bool LAST>
__device__ __forceinline__ LmChunk tile(const AttentionArgs& a, uint32_t rows, uint32_t rank, int lane) {
  if (a.n > kSorted) return lm_chunk(a.offsets, a.n, a.T, rows, LAST ? a.slots - 1 - rank : rank, lane);
  uint32_t tiles[kSorted / 64];
#pragma unroll
  for (int k = 0; k < kSorted / 64; ++k) {
    const int i = 64 * k + lane;
    tiles[k] = 0;
    if (i < a.n) {
      const int64_t o = lm_offset(a.offsets, i, a.T), e = lm_offset(a.offsets, i + 1, a.T);
      tiles[k] = e > o ? static_cast<uint32_t>(e - o + rows - 1) / rows : 0;
    }
  }
  const auto with = [&](uint32_t w) {
    uint32_t sum = 0;
#pragma unroll
    for (int k = 0; k < kSorted / 64; ++k) sum += tiles[k] >= w ? tiles[k] - w + 1 : 0;
    return lm_wave_sum(sum);
  };
  LmChunk c{0, 0, 0, 0};
  if (with(1) <= rank) return c;
  uint32_t step = 1, w = 1;
  while (with(2 * step) > rank) step *= 2;
  w = step;
  for (step /= 2; step; step /= 2)
    if (with(w + step) > rank) w += step;
  uint32_t left = rank - with(w + 1);      // among the tiles with w to pass, one in each of these sequences
#pragma unroll
  for (int k = 0; k < kSorted / 64; ++k) {
    const uint64_t these = __ballot(tiles[k] >= w);
    const uint32_t count = __builtin_popcountll(these);
    if (left < count) {
      const bool here = tiles[k] >= w && __builtin_popcountll(these & ((uint64_t{1} << lane) - 1)) == left;
      const int l = __builtin_ctzll(__ballot(here));
      c.group = 64 * k + l;
      const uint32_t j = LAST ? w - 1 : __builtin_amdgcn_readlane(tiles[k], l) - w;
      c.start = static_cast<int32_t>(lm_offset(a.offsets, c.group, a.T));
      c.end = static_cast<int32_t>(lm_offset(a.offsets, c.group + 1, a.T));
      c.first = static_cast<int32_t>(c.start + j * rows);
      break;
    }
    left -= count;
  }
  c.start = __builtin_amdgcn_readfirstlane(c.start);
  c.end = __builtin_amdgcn_readfirstlane(c.end);
  c.first = __builtin_amdgcn_readfirstlane(c.first);
  return c;
}
template <bool LAST>
__device__ __forceinline__ Work work(const AttentionArgs& a, uint32_t id, int heads, int rows, int lane) {
  return Work{tile<LAST>(a, rows, id / heads, lane), static_cast<int>(id % heads)};
}

// S groups of four waves, which take the same queries and every S-th 64 keys,
// and whose sums are joined at the end.
template <typename E, int DP, int S>
__global__ __launch_bounds__(256 * S, 2) void k_attention(AttentionArgs a) {
  typedef Rows<DP, BN * S, 256 * S> R;
  __shared__ __align__(16) char lds[4 * R::BYTES];   // two stages of K and V
  constexpr int VALUES = DP / 32 * 16 + 2;           // of a lane, to be joined
  static_assert(S == 1 || 4 * VALUES * 256 <= 4 * R::BYTES, "they go through LDS");
  const int tid = threadIdx.x, lane = tid % 64, all_waves = __builtin_amdgcn_readfirstlane(tid / 64);
  const int wave = all_waves % 4, part = all_waves / 4, c = lane % 32, h = lane / 32;
  lm_one_first();
  const Work w = work<true>(a, blockIdx.x, a.heads, BM, lane);
  if (w.rows.empty()) return;
  const int len = w.rows.end - w.rows.start, q0 = w.rows.first - w.rows.start, qw = q0 + 32 * wave, qi = qw + c;
  const int kv_head = w.head / (a.heads / a.kv_heads);
  const float scale2 = a.scale * kLog2E;
  const float lim = 8.f / scale2;    // a maximum may grow by 2^8 before sums are scaled
  bool far = false;                  // whether a maximum of the wave's lies beyond kFar
  const int64_t row = w.rows.first + int64_t{32} * wave;

  lm_u32x4 q[DP / 16];
  operand<DP>(at(a.Q, row, w.head), a.Q.token, len - qw, a.D, lane, q);
  f32x16 o[DP / 32];
#pragma unroll
  for (int i = 0; i < DP / 32; ++i) o[i] = zero16();
  float m = -INFINITY, sum = 0.f;

  uint32_t off_k[R::OFFSETS], off_v[R::OFFSETS], pv[DP / 32];
#pragma unroll
  for (int i = 0; i < R::OFFSETS; ++i) {
    off_k[i] = R::offset(a.K.token, BN * S, a.D, tid, i);
    off_v[i] = R::offset(a.V.token, BN * S, a.D, tid, i);
  }
  R::columns(lds + R::BYTES + part * (BN * DP * 2), lane, pv);
  const int keys = std::min(len, q0 + BM);   // the workgroup's
  const auto issue = [&](int k0, int slot) {
    char* to = lds + slot * (2 * R::BYTES);
    R::load(at(a.K, w.rows.start + static_cast<int64_t>(k0), kv_head), a.K.token, len - k0, a.D, to, all_waves, lane, off_k);
    R::load(at(a.V, w.rows.start + static_cast<int64_t>(k0), kv_head), a.V.token, len - k0, a.D, to + R::BYTES, all_waves, lane, off_v);
  };
  issue(0, 0);
  for (int first = 0, slot = 0; first < keys; first += BN * S, slot ^= 1) {
    wait_step<0>();
    if (first + BN * S < keys) issue(first + BN * S, slot ^ 1);
    const int k0 = first + BN * part;
    if (k0 > qw + 31 || qw >= len) continue;
    const char* stage = lds + slot * (2 * R::BYTES) + part * (BN * DP * 2);
    f32x16 s[2] = {zero16(), zero16()};
#pragma unroll
    for (int kk = 0; kk < DP / 16; ++kk)
#pragma unroll
      for (int t = 0; t < 2; ++t) s[t] = mma(R::row(stage, 32 * t, kk, lane), q[kk], s[t], E{});
    // six reads of keys on their way before the first product, and one more for
    // each (16384 tokens, 8 heads on 2 of 128: 576 -> 558 us; no gain for dQ and dK)
    __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
    for (int i = 0; i < DP / 8; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      if (i + 6 < DP / 8) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    if (k0 + BN - 1 > qw) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (k0 + 32 * t + place(r, h) > qi) s[t][r] = -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[t][r]);
    mx = max_halves(mx);
    if (__any(mx - m > lim)) {   // (a sum m + lim rounds by more than lim where m is large)
      const float top = fmaxf(m, mx), by = __builtin_amdgcn_exp2f((m - top) * scale2);
      m = top;
      sum *= by;
#pragma unroll
      for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] *= by;
      far = __any(!(fabsf(m * scale2) <= kFar));
    }
    if (far) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] -= m;
    }
    const float m2 = far ? 0.f : m * scale2;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[t][r] = __builtin_amdgcn_exp2f(fmaf(s[t][r], scale2, -m2));
        sum += s[t][r];
      }
    uint32_t p[DP / 32];
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) p[i] = pv[i] + slot * (2 * R::BYTES);
    lm_u32x4 v[DP / 32];
    const auto product = [&](auto tu) {
      constexpr int t = decltype(tu)::value / 2, u = decltype(tu)::value % 2;
      R::template column<(32 * t + 16 * u) * DP * 2>(p, v);
      const lm_u32x4 x = terms<E>(s[t], u);
#pragma unroll
      for (int i = 0; i < DP / 32; ++i) o[i] = mma(v[i], x, o[i], E{});
    };
    product(std::integral_constant<int, 0>{});
    product(std::integral_constant<int, 1>{});
    product(std::integral_constant<int, 2>{});
    product(std::integral_constant<int, 3>{});
  }
  sum = sum_halves(sum);
  if constexpr (S == 2) {
    // the second group's sums join the first's (it may have had no keys: its
    // maximum is then -infinity, and its share 0)
    float* to = reinterpret_cast<float*>(lds) + wave * VALUES * 64 + lane;
    wait_step<0>();
    if (part == 1) {
      to[0] = m;
      to[64] = sum;
#pragma unroll
      for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) to[(2 + i * 16 + r) * 64] = o[i][r];
    }
    wait_step<0>();
    if (part == 1) return;
    const float m1 = to[0], top = fmaxf(m, m1);
    const float by0 = __builtin_amdgcn_exp2f((m - top) * scale2), by1 = __builtin_amdgcn_exp2f((m1 - top) * scale2);
    m = top;
    sum = sum * by0 + to[64] * by1;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[i][r] = o[i][r] * by0 + to[(2 + i * 16 + r) * 64] * by1;
  }
  if (qw >= len) return;
  write_rows<E, DP>(at(a.O, row, w.head), a.O.token, len - qw, a.D, lane, o, 1.f / sum);
  if (a.lse && h == 0 && qi < len)
    a.lse[w.head * a.T + w.rows.start + qi] = fmaf(m, a.scale, __builtin_amdgcn_logf(sum) * kLn2);
}

// fp16 has no more than 2^-14 at its full precision, and P and dS of long rows lie
// around 2^-13 of a gradient: they are rounded, and multiplied, 2^kRaise times
// as large.  Where dS does not fit then (above 64), a wave goes on without.
// (8192 tokens in a row, gradients 0.02: dQ, dK and dV 1.5 times as far from 64
// bits as their own rounding without it.)
template <typename E>
constexpr int kRaise = std::is_same_v<E, _Float16> ? 10 : 0;
constexpr float kMostHalf = 65504.f;

// Whether a lane of the wave has a value above what fp16 holds.
__device__ __forceinline__ bool too_large(const f32x16& x) {
  float most = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(x[r]));
  return __any(most > kMostHalf);
}
template <int N>
__device__ __forceinline__ void times(f32x16 (&x)[N], float by) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) x[i][r] *= by;
}

template <typename E, int DP, int S>
__global__ __launch_bounds__(256 * S, 2) void k_attention_dq(AttentionArgs a) {
  typedef Rows<DP, BN * S, 256 * S> R;
  __shared__ __align__(16) char lds[4 * R::BYTES];   // two stages of K and V
  constexpr int VALUES = DP / 32 * 16;
  static_assert(S == 1 || 4 * VALUES * 256 <= 4 * R::BYTES, "the sums to be joined go through LDS");
  const int tid = threadIdx.x, lane = tid % 64, all_waves = __builtin_amdgcn_readfirstlane(tid / 64);
  const int wave = all_waves % 4, part = all_waves / 4, c = lane % 32, h = lane / 32;
  lm_one_first();
  const Work w = work<true>(a, blockIdx.x, a.heads, BM, lane);
  if (w.rows.empty()) return;
  const int len = w.rows.end - w.rows.start, q0 = w.rows.first - w.rows.start, qw = q0 + 32 * wave, qi = qw + c;
  const int kv_head = w.head / (a.heads / a.kv_heads);
  const float scale2 = a.scale * kLog2E;
  const int64_t row = w.rows.first + int64_t{32} * wave;

  lm_u32x4 q[DP / 16], dy[DP / 16];
  operand<DP>(at(a.Q, row, w.head), a.Q.token, len - qw, a.D, lane, q);
  operand<DP>(at(a.dO, row, w.head), a.dO.token, len - qw, a.D, lane, dy);
  const int64_t stats = w.head * a.T + w.rows.start, stat = stats + qi;
  // P = exp2((S - m) scale2 - lse2), with m = 0 unless a row of the workgroup's is
  // far from 0: lse, of one rounding, does not tell P there (see kFar), and maximum
  // and sum are formed again
  float all_lse[BM / 64];
#pragma unroll
  for (int i = 0; i < BM / 64; ++i) all_lse[i] = a.lse[stats + std::min(q0 + 64 * i + lane, len - 1)];
  const float own_lse = a.lse[stats + std::min(qi, len - 1)];
  float m = 0.f, lse2 = qi < len ? own_lse * kLog2E : 0.f;
  float delta = 0.f, raise = static_cast<float>(kRaise<E>);
  f32x16 dq[DP / 32];
#pragma unroll
  for (int i = 0; i < DP / 32; ++i) dq[i] = zero16();

  uint32_t off_k[R::OFFSETS], off_v[R::OFFSETS], pk[DP / 32];
#pragma unroll
  for (int i = 0; i < R::OFFSETS; ++i) {
    off_k[i] = R::offset(a.K.token, BN * S, a.D, tid, i);
    off_v[i] = R::offset(a.V.token, BN * S, a.D, tid, i);
  }
  R::columns(lds + part * (BN * DP * 2), lane, pk);
  const int keys = std::min(len, q0 + BM);
  const auto issue = [&](int k0, int slot) {
    char* to = lds + slot * (2 * R::BYTES);
    R::load(at(a.K, w.rows.start + static_cast<int64_t>(k0), kv_head), a.K.token, len - k0, a.D, to, all_waves, lane, off_k);
    R::load(at(a.V, w.rows.start + static_cast<int64_t>(k0), kv_head), a.V.token, len - k0, a.D, to + R::BYTES, all_waves, lane, off_v);
  };
  issue(0, 0);
  bool in_reach = true;
#pragma unroll
  for (int i = 0; i < BM / 64; ++i) in_reach &= fabsf(all_lse[i]) * kLog2E <= kFar;
  const bool far = !__all(in_reach);
  // one pass over the keys, the first stage on its way: for maximum and sum, for
  // delta alone, or for dQ
  enum Pass { SUM, DELTA, GRAD };
  const auto pass = [&](auto what, auto far_) {
    constexpr int WHAT = decltype(what)::value;
    constexpr bool FAR = decltype(far_)::value;
    float shift = (WHAT == DELTA ? 0.f : raise) - lse2;
    for (int first = 0, slot = 0; first < keys; first += BN * S, slot ^= 1) {
      wait_step<0>();
      if (first + BN * S < keys) issue(first + BN * S, slot ^ 1);
      const int k0 = first + BN * part;
      const char* stage = lds + slot * (2 * R::BYTES) + part * (BN * DP * 2);
      uint32_t p[DP / 32];
#pragma unroll
      for (int i = 0; i < DP / 32; ++i) p[i] = pk[i] + slot * (2 * R::BYTES);
      const auto half = [&](auto which) {
        constexpr int t = decltype(which)::value;
        const int k = k0 + 32 * t;
        if (k > qw + 31 || qw >= len) return;
        f32x16 s = zero16(), ds = zero16();
#pragma unroll
        for (int kk = 0; kk < DP / 16; ++kk) {
          s = mma(R::row(stage, 32 * t, kk, lane), q[kk], s, E{});
          if constexpr (WHAT != SUM) ds = mma(R::row(stage + R::BYTES, 32 * t, kk, lane), dy[kk], ds, E{});
        }
        if constexpr (WHAT == SUM) {
          float top = m;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            if (k + place(r, h) > qi) s[r] = -INFINITY;
            top = fmaxf(top, s[r]);
          }
          top = max_halves(top);
          delta *= __builtin_amdgcn_exp2f((m - top) * scale2);
#pragma unroll
          for (int r = 0; r < 16; ++r) delta += __builtin_amdgcn_exp2f((s[r] - top) * scale2);
          m = top;
          return;
        }
        if constexpr (FAR) s -= m;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          ds[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale2, shift)) * (WHAT == DELTA ? ds[r] : ds[r] - delta);
        if (k + 31 > qw) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (k + place(r, h) > qi) ds[r] = 0.f;
        }
        if constexpr (WHAT == DELTA) {
#pragma unroll
          for (int r = 0; r < 16; ++r) delta += ds[r];
        } else {
          if (kRaise<E> && raise > 0.f && too_large(ds)) {
            times(dq, 1.f / (1 << kRaise<E>));
            ds *= 1.f / (1 << kRaise<E>);
            raise = 0.f;
            shift = -lse2;
          }
          lm_u32x4 f[DP / 32];
          R::template column<32 * t * DP * 2>(p, f);
          const lm_u32x4 x0 = terms<E>(ds, 0), x1 = terms<E>(ds, 1);
#pragma unroll
          for (int i = 0; i < DP / 32; ++i) dq[i] = mma(f[i], x0, dq[i], E{});
          R::template column<(32 * t + 16) * DP * 2>(p, f);
#pragma unroll
          for (int i = 0; i < DP / 32; ++i) dq[i] = mma(f[i], x1, dq[i], E{});
        }
      };
      half(std::integral_constant<int, 0>{});
      half(std::integral_constant<int, 1>{});
    }
  };
  if (far) {
    m = -INFINITY;
    pass(std::integral_constant<int, SUM>{}, std::true_type{});
    float sum = sum_halves(delta);
    wait_step<0>();
    if constexpr (S == 2) {
      // (the second group may have had no keys)
      float* both = reinterpret_cast<float*>(lds) + lane;
      both[64 * all_waves] = m;
      both[64 * (all_waves + 8)] = sum;
      wait_step<0>();
      const float m0 = both[64 * wave], m1 = both[64 * (wave + 4)];
      m = fmaxf(m0, m1);
      sum = both[64 * (wave + 8)] * __builtin_amdgcn_exp2f((m0 - m) * scale2) +
            both[64 * (wave + 12)] * __builtin_amdgcn_exp2f((m1 - m) * scale2);
      wait_step<0>();
    }
    issue(0, 0);
    lse2 = __builtin_amdgcn_logf(sum);
    delta = 0.f;
  }
  if (q0 == 0) {
    // The first queries have few keys, their O is as large as V, and O's rounding
    // would move delta by as much as dS is rounded: they take delta = sum_s P (dO .
    // V), a pass over at most two stages of keys (dQ, dK and dV of 100 tokens in
    // bf16 1.48 times as far from 64 bits as their own rounding, 1.40 so).
    if (far) pass(std::integral_constant<int, DELTA>{}, std::true_type{});
    else pass(std::integral_constant<int, DELTA>{}, std::false_type{});
    delta = sum_halves(delta);
    wait_step<0>();
    if constexpr (S == 2) {
      float* both = reinterpret_cast<float*>(lds) + lane;
      both[64 * all_waves] = delta;
      wait_step<0>();
      delta = both[64 * wave] + both[64 * (wave + 4)];
      wait_step<0>();
    }
    issue(0, 0);
  } else {
    lm_u32x4 y[DP / 16];
    operand<DP>(at(a.O, row, w.head), a.O.token, len - qw, a.D, lane, y);
    typedef E V __attribute__((ext_vector_type(8)));
#pragma unroll
    for (int kk = 0; kk < DP / 16; ++kk) {
      const V x = __builtin_bit_cast(V, y[kk]), g = __builtin_bit_cast(V, dy[kk]);
#pragma unroll
      for (int j = 0; j < 8; ++j) delta = fmaf(lm_to_f32(x[j]), lm_to_f32(g[j]), delta);
    }
    delta = sum_halves(delta);
  }
  if (far) pass(std::integral_constant<int, GRAD>{}, std::true_type{});
  else pass(std::integral_constant<int, GRAD>{}, std::false_type{});
  if (h == 0 && part == 0 && qi < len) {
    const int64_t all = a.heads * a.T;
    a.delta[stat] = delta;
    a.delta[all + stat] = lse2 - kRaise<E>;
    a.delta[2 * all + stat] = m;
  }
  if (kRaise<E>) times(dq, raise > 0.f ? 1.f / (1 << kRaise<E>) : 1.f);
  if constexpr (S == 2) {
    float* to = reinterpret_cast<float*>(lds) + wave * VALUES * 64 + lane;
    wait_step<0>();
    if (part == 1)
#pragma unroll
      for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) to[(i * 16 + r) * 64] = dq[i][r];
    wait_step<0>();
    if (part == 1) return;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) dq[i][r] += to[(i * 16 + r) * 64];
  }
  if (qw >= len) return;
  write_rows<E, DP>(at(a.dQ, row, w.head), a.dQ.token, len - qw, a.D, lane, dq, a.scale);
}

// A lane's sums of a row (see write_rows), as they are.
template <int DP>
__device__ __forceinline__ void write_sums(float* row, int D, int lane, const f32x16 (&x)[DP / 32]) {
#pragma unroll
  for (int i = 0; i < DP / 32; ++i)
#pragma unroll
    for (int k = 0; k < 16; k += 4) {
      const int d = 32 * i + 2 * k + 4 * (lane / 32);
      if (d < D) *reinterpret_cast<lm_f32x4*>(row + d) = lm_f32x4{x[i][k], x[i][k + 1], x[i][k + 2], x[i][k + 3]};
    }
}

// Two groups of 32 keys, and each the G groups of 32 queries of a stage: 2 G
// waves, whose sums are joined at the end.  With a.parts > 1, as many workgroups
// have a part of the queries and heads each, and leave their sums to
// k_attention_join.
template <typename E, int DP, int G>
__global__ __launch_bounds__(128 * G, 2) void k_attention_dkv(AttentionArgs a) {
  constexpr int STEP = 32 * G, THREADS = 128 * G;
  typedef Rows<DP, STEP, THREADS> R;
  typedef Rows<DP, KEYS, THREADS> RV;
  // with 128 values a head, registers hold the keys but not the values beside the sums
  constexpr bool V_IN_LDS = DP == 128;
  constexpr int STAGE = 2 * R::BYTES + 2 * G * 256;      // Q, dO, and of each query: delta, lse, maximum (twice: every wave loads)
  constexpr int VALUES = DP / 32 * 2 * 16;           // sums of a lane
  __shared__ __align__(256) char lds[2 * STAGE + (V_IN_LDS ? KEYS * DP * 2 : 0)];
  static_assert(G * VALUES * 256 <= 2 * STAGE, "the sums of half the waves go through LDS");
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int c = lane % 32, h = lane / 32, part = wave / 2;
  lm_one_first();
  const Work w = work<false>(a, blockIdx.x / a.parts, a.kv_heads, KEYS, lane);
  if (w.rows.empty()) return;
  const int len = w.rows.end - w.rows.start, k0 = w.rows.first - w.rows.start, kw = k0 + 32 * (wave % 2), ki = kw + c;
  const int share = a.heads / a.kv_heads;
  const float scale2 = a.scale * kLog2E;
  const int64_t row = w.rows.first + int64_t{32} * (wave % 2);

  lm_u32x4 k[DP / 16], v[V_IN_LDS ? 1 : DP / 16];
  operand<DP>(at(a.K, row, w.head), a.K.token, len - kw, a.D, lane, k);
  if constexpr (V_IN_LDS) {
    uint32_t off[RV::OFFSETS];
#pragma unroll
    for (int i = 0; i < RV::OFFSETS; ++i) off[i] = RV::offset(a.V.token, KEYS, a.D, tid, i);
    RV::load(at(a.V, w.rows.first, w.head), a.V.token, len - k0, a.D, lds + 2 * STAGE, wave, lane, off);
  } else {
    operand<DP>(at(a.V, row, w.head), a.V.token, len - kw, a.D, lane, v);
  }
  f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
  for (int i = 0; i < DP / 32; ++i) dk[i] = dv[i] = zero16();
  bool raised = kRaise<E> > 0;

  uint32_t off_q[R::OFFSETS], off_d[R::OFFSETS], pq[DP / 32];
#pragma unroll
  for (int i = 0; i < R::OFFSETS; ++i) {
    off_q[i] = R::offset(a.Q.token, STEP, a.D, tid, i);
    off_d[i] = R::offset(a.dO.token, STEP, a.D, tid, i);
  }
  R::columns(lds + 32 * part * DP * 2, lane, pq);
  uint32_t line_q = 0, line_v = 0;
  if constexpr (V_IN_LDS) {
    line_q = R::line(lds, 32 * part, lane);
    line_v = RV::line(lds + 2 * STAGE, 32 * (wave % 2), lane);
  }
  // tiles of queries from the workgroup's first key on, for each head in turn
  const int steps = (len - k0 + STEP - 1) / STEP;
  const int64_t all = static_cast<int64_t>(steps) * share;
  const int piece = static_cast<int>(blockIdx.x % a.parts);
  const int64_t begin = all * piece / a.parts, end = all * (piece + 1) / a.parts;
  int head_of = static_cast<int>(begin / steps), q_of = k0 + static_cast<int>(begin % steps) * STEP;   // the next stage to load
  const auto issue = [&](int slot) {
    char* to = lds + slot * STAGE;
    const int head = w.head * share + head_of, left = len - q_of;
    const int64_t from = w.rows.start + static_cast<int64_t>(q_of);
    R::load(at(a.Q, from, head), a.Q.token, left, a.D, to, wave, lane, off_q);
    R::load(at(a.dO, from, head), a.dO.token, left, a.D, to + R::BYTES, wave, lane, off_d);
    typedef __attribute__((address_space(3))) void* P;
    const int i = wave % (G / 2) * 64 + lane;
    const int which = wave < G ? wave / (G / 2) : 2;
    const float* x = a.delta + (which * a.heads + head) * a.T + from;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(make_rsrc(x, static_cast<uint32_t>(kMaxBufferBytes)),
                                             (P)(to + 2 * R::BYTES + wave * 256), 4,
                                             i < left ? static_cast<uint32_t>(i * 4) : kOutOfRange, 0, 0, 0);
    q_of += STEP;
    if (q_of >= len) {
      q_of = k0;
      ++head_of;
    }
  };
  int q0 = q_of, slot = 0;
  if (begin < end) issue(0);
  for (int64_t i = begin; i < end; ++i, slot ^= 1) {
    wait_step<0>();
    if (i + 1 < end) issue(slot ^ 1);
    const int q = q0 + 32 * part;
    q0 += STEP;
    if (q0 >= len) q0 = k0;
    if (q + 31 < kw || q >= len || kw >= len) continue;
    const char* stage = lds + slot * STAGE;
    uint32_t p[DP / 32];
#pragma unroll
    for (int j = 0; j < DP / 32; ++j) p[j] = pq[j] + slot * STAGE;
    const char* stats = stage + 2 * R::BYTES + (32 * part + 4 * h) * 4;
    // whether one of 32 queries has a maximum, which is subtracted from whole sums: these
    // are then the same bits here as where the maximum is from
    const bool far = __any(*reinterpret_cast<const float*>(stage + 2 * R::BYTES + STEP * 8 + (32 * part + c) * 4) != 0.f);
    f32x16 s = zero16(), ds = zero16();
    if constexpr (V_IN_LDS) {
      const uint32_t at_q = line_q + slot * STAGE;
      asm("" : "+v"(line_v));   // (the addresses from it are not to be kept)
#pragma unroll
      for (int kk = 0; kk < DP / 16; ++kk) {
        s = mma(R::row(at_q, kk), k[kk], s, E{});
        ds = mma(R::row(at_q + R::BYTES, kk), RV::row(line_v, kk), ds, E{});
      }
    } else {
#pragma unroll
      for (int kk = 0; kk < DP / 16; ++kk) {
        s = mma(R::row(stage, 32 * part, kk, lane), k[kk], s, E{});
        ds = mma(R::row(stage + R::BYTES, 32 * part, kk, lane), v[kk], ds, E{});
      }
    }
    if (far) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const lm_f32x4 m = *reinterpret_cast<const lm_f32x4*>(stats + STEP * 8 + 32 * g);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[4 * g + j] -= m[j];
      }
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const lm_f32x4 delta = *reinterpret_cast<const lm_f32x4*>(stats + 32 * g);
      const lm_f32x4 lse2 = *reinterpret_cast<const lm_f32x4*>(stats + STEP * 4 + 32 * g);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = 4 * g + j;
        s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale2, -lse2[j]));
        ds[r] = s[r] * (ds[r] - delta[j]);
      }
    }
    if (q < kw + 31 || q + 31 >= len) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (ki > q + place(r, h) || q + place(r, h) >= len) s[r] = ds[r] = 0.f;
    }
    if constexpr (kRaise<E> > 0) {
      constexpr float by = 1.f / (1 << kRaise<E>);
      if (raised && too_large(ds)) {
        raised = false;
        times(dk, by);
        times(dv, by);
      }
      if (!raised) {
        s *= by;
        ds *= by;
      }
    }
    const auto product = [&](auto at_) {
      constexpr int u = decltype(at_)::value;
      lm_u32x4 f[DP / 32];
      R::template column<16 * u * DP * 2>(p, f);
      const lm_u32x4 y = terms<E>(ds, u);
#pragma unroll
      for (int j = 0; j < DP / 32; ++j) dk[j] = mma(f[j], y, dk[j], E{});
      R::template column<16 * u * DP * 2 + R::BYTES>(p, f);
      const lm_u32x4 x = terms<E>(s, u);
#pragma unroll
      for (int j = 0; j < DP / 32; ++j) dv[j] = mma(f[j], x, dv[j], E{});
    };
    product(std::integral_constant<int, 0>{});
    product(std::integral_constant<int, 1>{});
  }
  if (kRaise<E> > 0 && raised) {
    times(dk, 1.f / (1 << kRaise<E>));
    times(dv, 1.f / (1 << kRaise<E>));
  }
  // the sums of the upper half of the waves join the lower half's, until two are left
#pragma unroll
  for (int from = G; from >= 2; from /= 2) {
    wait_step<0>();
    if (wave >= from && wave < 2 * from) {
      float* to = reinterpret_cast<float*>(lds) + (wave - from) * VALUES * 64 + lane;
#pragma unroll
      for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          to[(i * 32 + r) * 64] = dk[i][r];
          to[(i * 32 + 16 + r) * 64] = dv[i][r];
        }
    }
    wait_step<0>();
    if (wave < from) {
      const float* of = reinterpret_cast<const float*>(lds) + wave * VALUES * 64 + lane;
#pragma unroll
      for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          dk[i][r] += of[(i * 32 + r) * 64];
          dv[i][r] += of[(i * 32 + 16 + r) * 64];
        }
    }
  }
  if (wave >= 2 || kw >= len) return;
  if (a.parts > 1) {
    if (ki >= len) return;
    const int64_t rows = a.T * a.kv_heads, to = (w.rows.start + static_cast<int64_t>(ki)) * a.kv_heads + w.head;
    write_sums<DP>(a.sums + (2 * piece * rows + to) * a.D, a.D, lane, dk);
    write_sums<DP>(a.sums + ((2 * piece + 1) * rows + to) * a.D, a.D, lane, dv);
    return;
  }
  write_rows<E, DP>(at(a.dK, row, w.head), a.dK.token, len - kw, a.D, lane, dk, a.scale);
  write_rows<E, DP>(at(a.dV, row, w.head), a.dV.token, len - kw, a.D, lane, dv, 1.f);
}

// dK and dV from the sums of their parts, in order; a thread takes eight values
// of a row.
template <typename E>
__global__ __launch_bounds__(256) void k_attention_join(AttentionArgs a) {
  const int chunks = a.D / 8;
  const int64_t first = lm_offset(a.offsets, 0, a.T), end = lm_offset(a.offsets, a.n, a.T);
  const int64_t all = (end - first) * a.kv_heads * chunks, values = a.T * a.kv_heads * a.D;
  const bool v = blockIdx.y == 1;
  const HeadRows& out = v ? a.dV : a.dK;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < all; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t at_ = first * a.kv_heads * chunks + i, row = at_ / chunks;
    const float* p = a.sums + (v ? values : 0) + at_ * 8;
    lm_f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
    for (int k = 0; k < a.parts; ++k, p += 2 * values) {
      x += *reinterpret_cast<const lm_f32x4*>(p);
      y += *reinterpret_cast<const lm_f32x4*>(p + 4);
    }
    const float by = v ? 1.f : a.scale;
    *reinterpret_cast<lm_u32x4*>(at(out, row / a.kv_heads, static_cast<int>(row % a.kv_heads)) + at_ % chunks * 16) =
        lm_u32x4{pack2<E>(x[0] * by, x[1] * by), pack2<E>(x[2] * by, x[3] * by), pack2<E>(y[0] * by, y[1] * by),
                 pack2<E>(y[2] * by, y[3] * by)};
  }
}

uint32_t slots_of(const AttentionArgs& a, int rows) { return static_cast<uint32_t>(a.T / rows + a.n); }

template <typename E, int DP, int S>
void launch_queries(const AttentionArgs& a, bool grad, hipStream_t s) {
  if (grad) k_attention_dq<E, DP, S><<<a.slots * a.heads, 256 * S, 0, s>>>(a);
  else k_attention<E, DP, S><<<a.slots * a.heads, 256 * S, 0, s>>>(a);
}
template <typename E, int DP>
void launch_typed(AttentionArgs a, bool grad, hipStream_t s) {
  a.slots = slots_of(a, BM);
  if (static_cast<int64_t>(a.slots) * a.heads <= kFewTiles) launch_queries<E, DP, 2>(a, grad, s);
  else launch_queries<E, DP, 1>(a, grad, s);
  if (!grad) return;
  a.slots = slots_of(a, KEYS);
  const uint32_t grid = a.slots * a.kv_heads * a.parts;
  if (DP == 128 || (grid <= kFewTiles && a.T / a.n >= 512)) k_attention_dkv<E, DP, 4><<<grid, 512, 0, s>>>(a);
  else k_attention_dkv<E, DP, DP == 128 ? 4 : 2><<<grid, 128 * (DP == 128 ? 4 : 2), 0, s>>>(a);
  if (a.parts > 1) {
    const int64_t blocks = (a.T * a.kv_heads * (a.D / 8) + 255) / 256;
    k_attention_join<E><<<dim3(static_cast<uint32_t>(std::min<int64_t>(blocks, 4096)), 2), 256, 0, s>>>(a);
  }
}
template <typename E>
void launch_wide(const AttentionArgs& a, bool grad, hipStream_t s) {
  if (a.D <= 64) launch_typed<E, 64>(a, grad, s);
  else if (a.D <= 96) launch_typed<E, 96>(a, grad, s);
  else launch_typed<E, 128>(a, grad, s);
}
hipError_t launch(AttentionArgs a, bool grad, hipStream_t s) {
  if (a.T == 0) return hipSuccess;
  if (a.dtype == DBW_BF16) launch_wide<__bf16>(a, grad, s);
  else launch_wide<_Float16>(a, grad, s);
  return hipGetLastError();
}

}  // namespace

// Parts of the queries of a tile of keys: until there are about four workgroups
// a CU, which then end within a quarter of the time of one another although
// the first keys of a sequence have all its queries to pass and the last ones
// none; with two steps of 128 queries at least.  us with 1 part, 512 / grid and
// 1024 / grid of them (joined): 1 sequence of 8192 tokens, 8 heads on 2 of 128 541,
// 541, 386; 1 of 4096, 16 heads on 2 of 96 490, 160, 155.
int attention_parts(int n, int64_t T, int heads, int kv_heads) {
  const int64_t grid = (T / KEYS + n) * kv_heads, steps = T / n / 256 * (heads / kv_heads);
  return static_cast<int>(std::max<int64_t>(1, std::min({int64_t{1024} / grid, steps / 2, int64_t{16}})));
}

hipError_t launch_attention(AttentionArgs a, hipStream_t s) { return launch(a, false, s); }
hipError_t launch_attention_grad(AttentionArgs a, hipStream_t s) { return launch(a, true, s); }

}  // namespace dbw
