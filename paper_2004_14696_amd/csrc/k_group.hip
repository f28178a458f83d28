// Products of ragged groups on the matrix cores: Y[t] = X[t] W_i,
// dX[t] = dY[t] W_i^T and G_i = sum over the rows of a group of X[t]^T dY[t].
//
// One kernel computes a tile of BM x BN outputs, BK terms of the sum a step.
// An operand is either contiguous along the sum (X, dY, and W in dX) or along
// the output (W in Y, both operands of G): the first is kept in LDS as lines
// of BK terms and read 16 bytes a lane, the second as it lies in memory, one
// line a term, and read with the transposing LDS load, so nothing is
// transposed beforehand.  Rows of another group, and what lies behind an edge,
// are zeros in LDS, in both operands: NaN and infinities there reach no sum.
//
// Steps are pipelined: while one is multiplied, the loads of the next STAGES -
// 1 are in flight, straight into LDS, with one barrier a step.  Two workgroups
// share a CU, so that one multiplies while the other waits, loads its first
// steps or stores (256 x 256 tiles, one workgroup a CU: 319 us where 128 x 256
// take 258, head 4096 x 1024 x 32000).
//
// What bounds it: long sums, the matrix cores at the clock they hold, busy 62%
// of the cycles, the rest LDS reads and barriers.  4096 rows, 16384 columns, bf16,
// TFLOP/s of Y, G and dX (a library product): 256 terms 670, 600, 540 (570); 1024
// 1030, 1050, 845 (1070); 4096 1310, 1370, 1155 (1370); 8192 1215, 1315, 1035
// (1390).  Head 4096 x 1024 x 32000 254 us, 1060 TFLOP/s.  Ragged groups, how evenly
// their tiles fall on the CUs: 32 groups (28 with rows) 8192 x 2048 x 1536 79 us, 650
// TFLOP/s and 3.0 TB/s.  G of short minibatches, its stores: 16 workers 8000 x 784 x
// 4000 78 us (200 MB; streamed past the caches 123 us became 107 for 32 groups, in
// pieces of 16 bytes instead of lines they had taken 163).  Few rows, the weights
// from memory: 16 groups (14 with rows) 37 x 2048 x 1408 16.5 us, 4.9 TB/s.
//
// v_mfma_f32_16x16x32 takes, in lane l = 16 g + c, row c and terms 8 g .. 8 g
// + 7 of each operand; its result r of a lane is row 4 g + r of the first
// operand, row c of the second.  The output's columns go in as the first
// operand, so a lane has four consecutive columns of one output row; they are
// turned into whole lines in LDS.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "dbw_buffer.h"
#include "lm_ops.h"

namespace dbw {
namespace {

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
  int k0, k1;
  int rows, cols;
  int line_a, line_b;   // values of a line of either matrix
};

// One operand's part of a step: L outputs x BK terms, by THREADS threads.
// SWAP: contiguous along the output, kept as it lies in memory, a line of L
// outputs for each term; else a line of BK terms for each output.
template <typename E, int L, int BK, int THREADS, bool SWAP>
struct Operand {
  static constexpr int CHUNKS = L * BK / 8 / THREADS;   // chunks of 16 bytes a thread
  static constexpr int LINE = (SWAP ? L : BK) / 8;      // chunks of a line
  static constexpr int STEP = THREADS / LINE;           // lines between a thread's chunks
  static constexpr int BYTES = L * BK * 2;
  static_assert(L * BK / 8 % THREADS == 0 && THREADS % LINE == 0, "whole chunks a thread");
  static_assert(BK == 64 || BK == 32, "turn() is for lines of eight or four chunks");

  // A line's chunks are turned by its number, so that the lanes that read
  // together meet in no bank: rows of 16 bytes at 16 outputs, or 8 bytes of
  // four terms r = 0..3 of two of the four groups of eight terms.
  static __device__ __forceinline__ int turn(int line) {
    if (SWAP) return (line & 3) << 1 | (L >= 128 ? ((line >> 3) & 1) << 3 : 0);
    return LINE == 8 ? line & 7 : (line >> 1) & 3;
  }

  // Line and chunk (of memory) that thread tid's chunk i of a stage holds.
  static __device__ __forceinline__ int line(int tid, int i) { return tid / LINE + i * STEP; }
  static __device__ __forceinline__ int chunk(int tid, int i) { return tid % LINE ^ turn(line(tid, i)); }

  // Byte offset in memory of chunk i from the first term of a step with `left`
  // terms, or one behind every buffer: such loads give 0.
  static __device__ __forceinline__ uint32_t offset(int64_t ld, int left, int length, int tid, int i) {
    const int at = line(tid, i), first = chunk(tid, i) * 8;
    const bool in = SWAP ? at < left && first < length : at < length && first < left;
    return in ? static_cast<uint32_t>((at * ld + first) * 2) : kOutOfRange;
  }

  // Fragments of a lane: terms 32 kk + 8 g .. + 7 of outputs first + 16 i + c,
  // of the stage AT bytes into LDS.
  template <int N, int AT>
  static __device__ __forceinline__ void fragments(const char* lds, int first, int kk, int lane, lm_u32x4 (&f)[N]) {
    const int c = lane % 16, g = lane / 16;
    if constexpr (SWAP) {
      // a transposing load takes, for each 16 lanes, four terms of 16 outputs:
      // lane 4 r + q gives the address of term r, outputs 4 q .. 4 q + 3, and
      // lane c gets the terms of output c; another takes the next four terms
      // (whose lines are turned alike)
      const int r = c / 4, q = c % 4, line = g * 8 + r;
      typedef __attribute__((address_space(3))) const char* P;
      uint32_t p[N];
#pragma unroll
      for (int i = 0; i < N; ++i)
        p[i] = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(
            (P)(lds + line * (L * 2) + (((first + 16 * i) / 8 + q / 2) ^ turn(line)) * 16 + q % 2 * 8)));
      lm_u32x2 x[N][2];
      if (kk == 0)
        read_turned<AT>(p, x);
      else
        read_turned<(BK == 64 ? AT + 32 * L * 2 : AT)>(p, x);
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = lm_u32x4{x[i][0][0], x[i][0][1], x[i][1][0], x[i][1][1]};
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int row = first + 16 * i + c;
        f[i] = *reinterpret_cast<const lm_u32x4*>(lds + AT + row * (BK * 2) + ((kk * 4 + g) ^ turn(row)) * 16);
      }
    }
  }

  // The transposing loads of N tiles, and the wait for them, in one statement:
  // as builtins, the compiler would first wait for every load on its way to LDS.
  template <int AT>
  static __device__ __forceinline__ void read_turned(const uint32_t (&p)[4], lm_u32x2 (&x)[4][2]) {
    static_assert(AT + 4 * L * 2 < 65536, "sixteen bits");
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
        "ds_read_b64_tr_b16 %2, %9 offset:%12\n\tds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
        "ds_read_b64_tr_b16 %4, %10 offset:%12\n\tds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
        "ds_read_b64_tr_b16 %6, %11 offset:%12\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]), "=&v"(x[2][1]),
          "=&v"(x[3][0]), "=&v"(x[3][1])
        : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "n"(AT), "n"(AT + 4 * L * 2)
        : "memory");
  }
  template <int AT>
  static __device__ __forceinline__ void read_turned(const uint32_t (&p)[8], lm_u32x2 (&x)[8][2]) {
    static_assert(AT + 4 * L * 2 < 65536, "sixteen bits");
    asm volatile(
        "ds_read_b64_tr_b16 %0, %16 offset:%24\n\tds_read_b64_tr_b16 %1, %16 offset:%25\n\t"
        "ds_read_b64_tr_b16 %2, %17 offset:%24\n\tds_read_b64_tr_b16 %3, %17 offset:%25\n\t"
        "ds_read_b64_tr_b16 %4, %18 offset:%24\n\tds_read_b64_tr_b16 %5, %18 offset:%25\n\t"
        "ds_read_b64_tr_b16 %6, %19 offset:%24\n\tds_read_b64_tr_b16 %7, %19 offset:%25\n\t"
        "ds_read_b64_tr_b16 %8, %20 offset:%24\n\tds_read_b64_tr_b16 %9, %20 offset:%25\n\t"
        "ds_read_b64_tr_b16 %10, %21 offset:%24\n\tds_read_b64_tr_b16 %11, %21 offset:%25\n\t"
        "ds_read_b64_tr_b16 %12, %22 offset:%24\n\tds_read_b64_tr_b16 %13, %22 offset:%25\n\t"
        "ds_read_b64_tr_b16 %14, %23 offset:%24\n\tds_read_b64_tr_b16 %15, %23 offset:%25\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]), "=&v"(x[2][1]),
          "=&v"(x[3][0]), "=&v"(x[3][1]), "=&v"(x[4][0]), "=&v"(x[4][1]), "=&v"(x[5][0]), "=&v"(x[5][1]),
          "=&v"(x[6][0]), "=&v"(x[6][1]), "=&v"(x[7][0]), "=&v"(x[7][1])
        : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "v"(p[4]), "v"(p[5]), "v"(p[6]), "v"(p[7]), "n"(AT),
          "n"(AT + 4 * L * 2)
        : "memory");
  }
};

// 16 bytes a lane from r + off to the wave's 1 KiB at `to`.
__device__ __forceinline__ void load_lds(__amdgpu_buffer_rsrc_t r, char* to, uint32_t off) {
  typedef __attribute__((address_space(3))) void* P;
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (P)to, 16, off, 0, 0, 0);
}

// Loads of one step after the other straight into LDS: a wave's instruction
// fills 1 KiB, lane by lane.  Needs whole chunks: every line of memory starts
// and ends at one.
template <typename Op, typename E, int BK, bool SWAP>
struct Direct {
  static constexpr int WAVES = Op::STEP * Op::LINE / 64;
  const E* p;                  // the next step's first term
  int64_t ld, step;
  int length;
  uint32_t off[Op::CHUNKS];
  __device__ __forceinline__ Direct(const E* first, int64_t ld_, int length_, int k0, int tid)
      : p(SWAP ? first + k0 * ld_ : first + k0), ld(ld_), step(SWAP ? BK * ld_ : BK), length(length_) {
#pragma unroll
    for (int i = 0; i < Op::CHUNKS; ++i) off[i] = Op::offset(ld, BK, length, tid, i);
  }
  // `left` terms from the step's first on: also 0 or fewer, behind the last
  // step, so that every step counts the same loads
  __device__ __forceinline__ void load(int left, char* lds, int wave, int lane) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(p, static_cast<uint32_t>(kMaxBufferBytes));
    if (left >= BK) {
#pragma unroll
      for (int i = 0; i < Op::CHUNKS; ++i) load_lds(r, lds + (i * WAVES + wave) * 1024, off[i]);
    } else {
#pragma unroll
      for (int i = 0; i < Op::CHUNKS; ++i)
        load_lds(r, lds + (i * WAVES + wave) * 1024, Op::offset(ld, left, length, wave * 64 + lane, i));
    }
    p += step;
  }
};

// v >> 16 s, for s in 1 .. 7.
__device__ __forceinline__ lm_u32x4 shift_halves(const lm_u32x4& v, int s) {
  uint64_t lo = v[0] | static_cast<uint64_t>(v[1]) << 32, hi = v[2] | static_cast<uint64_t>(v[3]) << 32;
  if (s >= 4) {
    lo = hi;
    hi = 0;
  }
  const int r = 16 * (s & 3);
  if (r) {
    lo = lo >> r | hi << (64 - r);
    hi >>= r;
  }
  return lm_u32x4{static_cast<uint32_t>(lo), static_cast<uint32_t>(lo >> 32), static_cast<uint32_t>(hi),
                  static_cast<uint32_t>(hi >> 32)};
}

// Loads of one step after the other through registers, for lines at any
// address and of any length.  A chunk that a line ends in is the line's last
// eight values, shifted when it goes to LDS: as many loads as whole chunks
// take, and no branch around any.  `total` values make a line of the matrix.
template <typename Op, typename E, int BK, bool SWAP>
struct Staged {
  const E* p;                  // eight values before the next step's first term
  int64_t ld, step;
  int length, total;
  int shift, end;              // of the step held: values that the last chunk lacks, its first place
  uint32_t off[Op::CHUNKS];
  lm_u32x4 held[Op::CHUNKS];
  __device__ __forceinline__ uint32_t offset(int left, int tid, int i) const {
    const int at = Op::line(tid, i), first = Op::chunk(tid, i) * 8, in_line = SWAP ? length : left;
    if (at >= (SWAP ? left : length) || first >= in_line) return kOutOfRange;
    return static_cast<uint32_t>((at * ld + 8 + (first + 8 <= in_line ? first : in_line - 8)) * 2);
  }
  __device__ __forceinline__ Staged(const E* first, int64_t ld_, int length_, int total_, int k0, int tid)
      : p((SWAP ? first + k0 * ld_ : first + k0) - 8), ld(ld_), step(SWAP ? BK * ld_ : BK), length(length_),
        total(total_) {
#pragma unroll
    for (int i = 0; i < Op::CHUNKS; ++i) off[i] = offset(BK, tid, i);
  }
  __device__ __forceinline__ void load(int left, int tid) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(p, static_cast<uint32_t>(kMaxBufferBytes));
    const int in_line = SWAP ? length : left;
    shift = 0;
    if (total >= 8) {
      if (in_line < Op::LINE * 8) {
        shift = -in_line & 7;
        end = in_line & ~7;
      }
      if (left >= BK) {
#pragma unroll
        for (int i = 0; i < Op::CHUNKS; ++i)
          held[i] = __builtin_bit_cast(lm_u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off[i], 0, 0));
      } else {
#pragma unroll
        for (int i = 0; i < Op::CHUNKS; ++i)
          held[i] = __builtin_bit_cast(lm_u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, offset(left, tid, i), 0, 0));
      }
    } else {
      // a matrix of fewer than eight columns: value by value
#pragma unroll
      for (int i = 0; i < Op::CHUNKS; ++i) {
        const int at = Op::line(tid, i), first = Op::chunk(tid, i) * 8;
#pragma unroll
        for (int j = 0; j < 4; ++j) held[i][j] = 0;
#pragma unroll
        for (int j = 0; j < 7; ++j) {
          const bool in = at < (SWAP ? left : length) && first + j < in_line;
          const uint32_t x = __builtin_amdgcn_raw_buffer_load_b16(
              r, in ? static_cast<uint32_t>((at * ld + 8 + first + j) * 2) : kOutOfRange, 0, 0);
          held[i][j / 2] |= (x & 0xffffu) << (16 * (j % 2));
        }
      }
    }
    p += step;
  }
  __device__ __forceinline__ void store(char* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < Op::CHUNKS; ++i) {
      lm_u32x4 v = held[i];
      if (shift) {
        const lm_u32x4 w = shift_halves(v, shift);
        v = Op::chunk(tid, i) * 8 == end ? w : v;
      }
      *reinterpret_cast<lm_u32x4*>(lds + (i * Op::STEP * Op::LINE + tid) * 16) = v;
    }
  }
};

// Waits until at most `loads` of this wave's loads are outstanding and all its
// LDS reads are done, then for the other waves.
template <int loads>
__device__ __forceinline__ void wait_step() {
  static_assert(loads < 64, "six bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((loads & 15) | 7 << 4 | 0 << 8 | (loads >> 4) << 14);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <typename E>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef float F __attribute__((ext_vector_type(2)));
  typedef E V __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(F{a, b}, V));
}

// N consecutive outputs of one row, `left` of them inside.
template <typename O, int N, bool STREAM = false>
__device__ __forceinline__ void store_out(O* p, const lm_u32x4& v, int left) {
  if (left >= N) {
    if (STREAM)
      __builtin_nontemporal_store(v, reinterpret_cast<lm_u32x4_any*>(p));
    else
      *reinterpret_cast<lm_u32x4_any*>(p) = v;
  } else {
    typedef O V __attribute__((ext_vector_type(N)));
    const V x = __builtin_bit_cast(V, v);
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < left) p[j] = x[j];
  }
}

// A wave's outputs, by way of its part of LDS: a lane has four columns of one
// row, memory takes whole lines.  Chunks of 16 bytes are turned by their row,
// as the operands' are.
template <typename O, int WM, int WN, int LDS, bool STREAM>
__device__ __forceinline__ void write_out(const f32x4 (&acc)[WM / 16][WN / 16], const Tile& t, int m0, int n0, char* lds,
                                          int lane) {
  constexpr int BYTES = WN * sizeof(O), CH = BYTES / 16, N = 16 / sizeof(O);
  constexpr int TILES = LDS / BYTES / 16 >= WM / 16 ? WM / 16 : LDS / BYTES >= 64 ? 4 : LDS / BYTES >= 32 ? 2 : 1;
  constexpr int ROWS = 16 * TILES;                     // rows of a pass
  static_assert(ROWS * BYTES <= LDS && WM % ROWS == 0 && ROWS * CH % 64 == 0, "whole passes");
  const int c = lane % 16, g = lane / 16;
#pragma unroll
  for (int p = 0; p < WM / ROWS; ++p) {
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      const int row = i * 16 + c;
#pragma unroll
      for (int j = 0; j < WN / 16; ++j) {
        const f32x4 x = acc[p * TILES + i][j];
        if constexpr (sizeof(O) == 4) {
          *reinterpret_cast<f32x4*>(lds + row * BYTES + ((j * 4 + g) ^ (row & (CH - 1) & 15)) * 16) = x;
        } else {
          *reinterpret_cast<lm_u32x2*>(lds + row * BYTES + ((j * 2 + g / 2) ^ (row & (CH - 1) & 15)) * 16 + g % 2 * 8) =
              lm_u32x2{pack2<O>(x[0], x[1]), pack2<O>(x[2], x[3])};
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < ROWS * CH / 64; ++i) {
      const int row = (i * 64 + lane) / CH, q = (i * 64 + lane) % CH;
      const lm_u32x4 v = *reinterpret_cast<const lm_u32x4*>(lds + row * BYTES + (q ^ (row & (CH - 1) & 15)) * 16);
      const int m = m0 + p * ROWS + row, n = n0 + q * N;
      if (m < t.rows && n < t.cols) store_out<O, N, STREAM>(static_cast<O*>(t.out) + m * t.ldo + n, v, t.cols - n);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

template <typename E, int BM, int BN, int WM, int WN, int BK, int STAGES, bool A_SWAP, bool B_SWAP, bool WIDE,
          bool STREAM>
__device__ __forceinline__ void product(const Tile& t, bool out_f32, char* lds) {
  constexpr int THREADS = (BM / WM) * (BN / WN) * 64;
  constexpr int TM = WM / 16, TN = WN / 16;
  typedef Operand<E, BM, BK, THREADS, A_SWAP> OpA;
  typedef Operand<E, BN, BK, THREADS, B_SWAP> OpB;
  constexpr int STAGE = OpA::BYTES + OpB::BYTES;
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int m0 = wave / (BN / WN) * WM, n0 = wave % (BN / WN) * WN;
  const E* a = static_cast<const E*>(t.a);
  const E* b = static_cast<const E*>(t.b);

  f32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const auto multiply = [&](const char* stages, auto slot) {
    constexpr int AT = decltype(slot)::value * STAGE;
#pragma unroll
    for (int kk = 0; kk < BK / 32; ++kk) {
      lm_u32x4 fa[TM], fb[TN];
      OpA::template fragments<TM, AT>(stages, m0, kk, lane, fa);
      OpB::template fragments<TN, AT + OpA::BYTES>(stages, n0, kk, lane, fb);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mma(fb[j], fa[i], acc[i][j], E{});
    }
  };

  if constexpr (WIDE) {
    Direct<OpA, E, BK, A_SWAP> A(a, t.lda, t.rows, t.k0, tid);
    Direct<OpB, E, BK, B_SWAP> B(b, t.ldb, t.cols, t.k0, tid);
    const auto issue = [&](int left, int slot) {
      A.load(left, lds + slot * STAGE, wave, lane);
      B.load(left, lds + slot * STAGE + OpA::BYTES, wave, lane);
    };
    int left = t.k1 - t.k0;      // terms from the present step on
    if (left > 0) {
#pragma unroll
      for (int s = 0; s < STAGES - 1; ++s) issue(left - s * BK, s);
      // the slots in turn, each with its own code: their places are constants
      const auto step = [&](auto slot) {
        constexpr int SLOT = decltype(slot)::value;
        // this step's loads have landed, and nobody reads the slot of the step
        // before any more
        wait_step<(STAGES - 2) * (OpA::CHUNKS + OpB::CHUNKS)>();
        issue(left - (STAGES - 1) * BK, (SLOT + STAGES - 1) % STAGES);
        multiply(lds, slot);
        left -= BK;
      };
      for (;;) {
        step(std::integral_constant<int, 0>{});
        if (left <= 0) break;
        step(std::integral_constant<int, 1>{});
        if (left <= 0) break;
        if constexpr (STAGES > 2) {
          step(std::integral_constant<int, 2>{});
          if (left <= 0) break;
        }
        if constexpr (STAGES > 3) {
          step(std::integral_constant<int, 3>{});
          if (left <= 0) break;
        }
      }
      // nothing may land in LDS any more: the outputs go through it
      wait_step<0>();
    }
  } else {
    Staged<OpA, E, BK, A_SWAP> A(a, t.lda, t.rows, t.line_a, t.k0, tid);
    Staged<OpB, E, BK, B_SWAP> B(b, t.ldb, t.cols, t.line_b, t.k0, tid);
    int left = t.k1 - t.k0;
    const auto load = [&](int of) {
      A.load(of, tid);
      B.load(of, tid);
    };
    const auto store = [&](int slot) {
      A.store(lds + slot * STAGE, tid);
      B.store(lds + slot * STAGE + OpA::BYTES, tid);
      __syncthreads();
    };
    if (left > 0) {
      load(left);
      store(0);
      for (int slot = 0; left > 0; slot ^= 1, left -= BK) {
        if (left > BK) load(left - BK);
        multiply(lds + slot * STAGE, std::integral_constant<int, 0>{});
        if (left > BK) store(slot ^ 1);
      }
    }
    __syncthreads();   // the outputs go through LDS
  }

  constexpr int LDS = (WIDE ? STAGES : 2) * STAGE / (THREADS / 64);   // bytes a wave
  char* mine = lds + wave * LDS;
  if (out_f32)
    write_out<float, WM, WN, LDS, STREAM>(acc, t, m0, n0, mine, lane);
  else
    write_out<E, WM, WN, LDS, STREAM>(acc, t, m0, n0, mine, lane);
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
  uint32_t row_tiles, col_tiles, blocks, run;
  int out_f32, out_bytes;
};

// Terms of one part of a sum of `length` terms: whole steps.
__device__ __forceinline__ int64_t split_of(int64_t length, int splits) {
  return ((length + 63) / 64 + splits - 1) / splits * 64;
}

template <typename E, int BM, int BN, int WM, int WN, int BK, int STAGES, int FORM, bool WIDE>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64, 2) void k_group(GroupArgs g) {
  constexpr bool A_SWAP = FORM == DBW_GROUP_WEIGHT_GRAD, B_SWAP = FORM != DBW_GROUP_INPUT_GRAD;
  __shared__ __align__(16) char lds[(WIDE ? STAGES : 2) * (BM + BN) * BK * 2];
  // Workgroups go to the eight XCDs in turn; consecutive tiles share an
  // operand, so each XCD (and its L2) takes runs of them: g.run of every 8
  // g.run, which spreads large and small groups over all XCDs.
  const uint32_t id = blockIdx.x / (8 * g.run) * (8 * g.run) + blockIdx.x % 8 * g.run + blockIdx.x % (8 * g.run) / 8;
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
    t.line_a = g.d;
    t.line_b = g.C;
    t.k0 = static_cast<int>(first + std::min<int64_t>(length, split * step));
    t.k1 = static_cast<int>(first + std::min<int64_t>(length, (split + 1) * step));
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
    t.line_a = K;
    t.line_b = g.C;
    t.a = static_cast<const E*>(g.a) + row * t.lda;
    t.b = static_cast<const E*>(g.b) + group * g.st_W + (FORM == DBW_GROUP_FORWARD ? n : n * g.ld_W);
    t.k0 = static_cast<int>(std::min<int64_t>(K, split * step));
    t.k1 = static_cast<int>(std::min<int64_t>(K, (split + 1) * step));
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
  product<E, BM, BN, WM, WN, BK, STAGES, A_SWAP, B_SWAP, WIDE, FORM == DBW_GROUP_WEIGHT_GRAD>(t, g.splits > 1 || g.out_f32, lds);
}

// out = the sum of the partial outputs, in the order of the parts; a thread
// takes four columns of a row.
template <typename O>
__global__ __launch_bounds__(256) void k_group_sum(GroupArgs g, const float* __restrict__ parts) {
  const bool grad = g.form == DBW_GROUP_WEIGHT_GRAD;
  const uint32_t N = g.form == DBW_GROUP_INPUT_GRAD ? g.d : g.C, quads = (N + 3) / 4;
  // rows outside the groups stay as they were
  const uint32_t first = grad ? 0 : static_cast<uint32_t>(lm_offset(g.offsets, 0, g.T));
  const uint32_t end = grad ? static_cast<uint32_t>(g.n) * g.d : static_cast<uint32_t>(lm_offset(g.offsets, g.n, g.T));
  if (end <= first) return;
  // (a split product has fewer than 512 tiles of outputs: 32 bits hold them)
  const uint32_t all = (end - first) * quads;
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += gridDim.x * 256) {
    const uint32_t row = first + i / quads, n = i % quads * 4;
    const float* p = parts + static_cast<int64_t>(row) * N + n;
    const int left = N - n < 4 ? static_cast<int>(N - n) : 4;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    if (left == 4) {
#pragma unroll 8
      for (int s = 0; s < g.splits; ++s) x += *reinterpret_cast<const lm_f32x4_any*>(p + s * g.part);
    } else {
      for (int s = 0; s < g.splits; ++s)
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (j < left) x[j] += p[s * g.part + j];
    }
    O* q = static_cast<O*>(g.out) +
           (grad ? row / g.d * g.st_W + row % g.d * g.ld_W : row * (g.form == DBW_GROUP_FORWARD ? g.ld_C : g.ld_d)) + n;
    if constexpr (std::is_same_v<O, float>) {
      store_out<float, 4>(q, __builtin_bit_cast(lm_u32x4, x), left);
    } else {
      const lm_u32x2 v = {pack2<O>(x[0], x[1]), pack2<O>(x[2], x[3])};
      if (left == 4) {
        *reinterpret_cast<lm_u32x2_any*>(q) = v;
      } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (j < left) q[j] = static_cast<O>(x[j]);
      }
    }
  }
}

enum GroupVariant { SMALL = 0, MIDDLE = 1, LARGE = 2 };
struct VariantSize {
  int bm, bn;
};
constexpr VariantSize kSize[] = {{32, 128}, {128, 128}, {128, 256}};

template <typename E, int FORM, bool WIDE>
void launch_variant(const GroupPlan& plan, const GroupArgs& g, uint32_t grid, hipStream_t s) {
  constexpr bool GRAD = FORM == DBW_GROUP_WEIGHT_GRAD;
  constexpr int BK = WIDE && GRAD ? 32 : 64;
  if constexpr (WIDE && FORM != DBW_GROUP_INPUT_GRAD)
    if (plan.variant == LARGE) {
      k_group<E, 128, 256, 64, 128, 32, 3, FORM, WIDE><<<grid, 256, 0, s>>>(g);
      return;
    }
  if constexpr (!GRAD)
    if (plan.variant == SMALL) {
      k_group<E, 32, 128, 16, 64, 64, 3, FORM, WIDE><<<grid, 256, 0, s>>>(g);
      return;
    }
  k_group<E, 128, 128, 64, 64, BK, 128 / BK, FORM, WIDE><<<grid, 256, 0, s>>>(g);
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

namespace {

// The plan with a given variant and number of parts of the sum.
GroupPlan plan_of(const dbw_group_shape& p, int variant, int splits) {
  GroupPlan plan;
  const bool grad = p.form == DBW_GROUP_WEIGHT_GRAD;
  const int64_t groups = p.st_W == 0 && !grad ? 1 : p.n;
  const int64_t N = p.form == DBW_GROUP_INPUT_GRAD ? p.d : p.C;
  const int64_t rows = grad ? p.d : std::max<int64_t>(1, p.T / groups);   // of one group, on average
  const VariantSize size = kSize[variant];
  plan.variant = variant;
  // every group may end in a tile of its own
  plan.row_tiles = grad ? ceil_div(p.d, size.bm)
                        : std::min<int64_t>(p.T, p.T / size.bm + std::min<int64_t>(groups, p.T));
  plan.col_tiles = ceil_div(N, size.bn);
  plan.tiles = std::max<int64_t>(1, ceil_div(rows, size.bm) * plan.col_tiles * groups);
  plan.splits = splits;
  plan.part = grad ? static_cast<int64_t>(p.n) * p.d * p.C : p.T * N;
  plan.blocks = plan.row_tiles * plan.col_tiles * plan.splits * (grad ? p.n : 1);
  return plan;
}

// Terms of the sum, on average.
int64_t terms(const dbw_group_shape& p) {
  return p.form == DBW_GROUP_WEIGHT_GRAD ? p.T / p.n : p.form == DBW_GROUP_FORWARD ? p.d : p.C;
}

// The best plan of a variant for Y and dX, by an estimate of its time in us:
//   steps of 64 terms, whose time was measured with one workgroup on a CU and
//   with two (1 x 1024 x 1024 x 1024 and 1 x 2048 x 1024 x 1024 with 32 x 128, 1 x 4096 x
//   1024 x 4096 and x 8192 with 128 x 128), for as many rounds as the tiles of
//   ragged groups take;
//   or the weights' way from memory, once for every row tile, where they are
//   larger than caches hold beside the rest (16 groups of 16 and 64 rows 2048 x 2048: 27 us with
//   32 x 128 and 50 against 39 us with 128 x 128);
//   and the sum of the parts: a launch, and the parts written and read.
struct Estimate {
  GroupPlan plan;
  double us;
};
Estimate best_plan(const dbw_group_shape& p, int variant) {
  const bool small = variant == SMALL;
  const double one = small ? 0.33 : 0.75, two = small ? 0.53 : 1.05;   // us a step
  Estimate best{plan_of(p, variant, 1), 0.0};
  const double groups = p.st_W == 0 ? 1 : p.n, rows = p.T / groups;
  // a group ends, on average, in the middle of a tile
  const double row_tiles = groups > 1 ? std::max(1.0, rows / kSize[variant].bm + 0.5)
                                      : static_cast<double>(ceil_div(p.T, kSize[variant].bm));
  const double tiles = groups * row_tiles * best.plan.col_tiles, K = static_cast<double>(terms(p));
  const double weights = 2.0 * groups * p.d * p.C, traffic = weights > 64e6 ? weights * row_tiles : 0.0;
  const int most = static_cast<int>(std::max(1.0, std::min({512 / tiles, K / 256, 64.0})));
  for (int s = 1; s <= most; ++s) {
    const double blocks = tiles * s, rounds = blocks <= 512 ? 1.0 : std::ceil(blocks / 512);
    const double step = blocks <= 256 ? one : two * rounds;
    const double rate = small ? 5.0e6 * std::min(1.0, blocks / 192) : blocks <= 256 ? 3.0e6 : 4.5e6;   // bytes a us
    const double sum = s > 1 ? 5.0 + 0.2 * s + 1e-6 * s * best.plan.part : 0.0;
    const double us = std::max(K / 64 / s * step, traffic / rate) + sum;
    if (s == 1 || us < best.us) best = Estimate{plan_of(p, variant, s), us};
  }
  return best;
}

// The parts of G's sums in 128 x 128 tiles, by an estimate of the time in us:
// steps of 64 terms, with one workgroup on a CU and with two, and what the parts
// cost: a launch, their loads (eight under way at once) and every workgroup's
// part written and read; where the lines are whole chunks, and where not.
// Fitted to 2 to 256 tiles with 2048, 8192 and 30000 terms (and 1024 in odd
// widths) in 1 to 64 parts; of the parts timed, its choice took at most 17% more
// than the fastest.
// Neither one nor two workgroups a CU is best throughout (us for 256 and for 512
// workgroups): 2048 terms 64 tiles 21 and 24, 192 tiles 25 and 30; 8192 terms 24
// tiles 20 and 23, 64 tiles 32 and 30, 128 tiles 53 and 43; 30000 terms 32 tiles 49
// and 41, 64 tiles 87 and 66, 128 tiles 166 and 137.
int weight_grad_parts(const dbw_group_shape& p, int64_t tiles) {
  const bool whole = p.d % 8 == 0 && p.C % 8 == 0 && p.ld_d % 8 == 0 && p.ld_C % 8 == 0;
  const double one = whole ? 0.60 : 1.27, two = whole ? 0.88 : 1.57;
  const double launch = whole ? 3.3 : 4.4, load = whole ? 0.17 : 0.90, block = whole ? 0.0145 : 0.026;
  const int64_t length = terms(p);
  const int most = static_cast<int>(std::min<int64_t>({512 / tiles, length / 256, 64}));
  int best = 1;
  double best_us = 0.0;
  for (int s = 1; s <= most; ++s) {
    const int64_t blocks = tiles * s, steps = ceil_div(ceil_div(length, 64), s);
    const double us = steps * (blocks <= 256 ? one : two) + (s > 1 ? launch + load * (s / 8 + s % 8) + block * blocks : 0.0);
    if (s == 1 || us < best_us) {
      best = s;
      best_us = us;
    }
  }
  return best;
}

}  // namespace

GroupPlan group_plan(const dbw_group_shape& p) {
  if (p.form == DBW_GROUP_WEIGHT_GRAD) {
    // 128 x 256: more products a value read, from one and a half tiles a CU on
    // (1 x 4096 x 1024 x 8192: 81 us either way; 32 groups 8192 x 2048 x 1536: 104
    // against 121 us).  Below, parts of the sum, each with 256 terms at least.
    if (const GroupPlan large = plan_of(p, LARGE, 1); large.tiles >= 384) return large;
    return plan_of(p, MIDDLE, weight_grad_parts(p, plan_of(p, MIDDLE, 1).tiles));
  }
  // Y in tiles of 128 x 256 from one and a half a CU on (1 x 4096 x 1024 x 4096, 512
  // tiles: 37 against 47 us; 1 x 2560 x 1024 x 4096, 320 tiles: 32 against 33 us; 1 x
  // 4096 x 1024 x 2048, 256 tiles: 25 against 23 us).  Not dX: both operands are
  // read in lines of the sum there, which 32 terms a step cut in halves (32
  // groups 8192 x 2048 x 1536: 85 against 75 us).
  const int64_t groups = p.st_W == 0 ? 1 : p.n;
  if (const GroupPlan large = plan_of(p, LARGE, 1);
      p.form == DBW_GROUP_FORWARD && large.tiles >= 384 && p.T / groups > 32)
    return large;
  // 32 x 128 for groups of few rows, which a taller tile would mostly leave
  // empty (16 groups of 2 rows 2048 x 1408: 19 against 22 us), and where it is
  // estimated to take less time.
  const Estimate small = best_plan(p, SMALL), middle = best_plan(p, MIDDLE);
  return p.T / groups <= 32 || small.us <= middle.us ? small.plan : middle.plan;
}

hipError_t launch_group(const dbw_group_shape& p, GroupPlan plan, const int32_t* offsets, const void* a,
                        const void* b, void* out, float* workspace, hipStream_t s) {
  const bool grad = p.form == DBW_GROUP_WEIGHT_GRAD;
  if (!grad && p.T == 0) return hipSuccess;
  // whole chunks of 16 bytes: every row starts at one and ends with one
  const auto even = [](const void* q, int64_t ld) { return reinterpret_cast<uintptr_t>(q) % 16 == 0 && ld % 8 == 0; };
  bool wide = p.d % 8 == 0 && p.C % 8 == 0;
  if (p.form == DBW_GROUP_FORWARD)
    wide = wide && even(a, p.ld_d) && even(b, p.ld_W) && p.st_W % 8 == 0;
  else if (p.form == DBW_GROUP_INPUT_GRAD)
    wide = wide && even(a, p.ld_C) && even(b, p.ld_W) && p.st_W % 8 == 0;
  else
    wide = wide && even(a, p.ld_d) && even(b, p.ld_C);
  // (the large tile is for whole chunks; its plan has no parts either)
  if (!wide && plan.variant == LARGE) plan = plan_of(p, MIDDLE, 1);
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
  g.run = std::min((g.blocks + 7) / 8, 32u);
  const uint32_t grid = static_cast<uint32_t>(ceil_div(g.blocks, 8 * g.run)) * 8 * g.run;
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
