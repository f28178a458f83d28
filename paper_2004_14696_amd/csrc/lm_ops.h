// Internal declarations of the operators for language models: grouped
// products, token loss, AdamW, and those of a transformer block.  Not part of the C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>
#include <type_traits>

#include "dbw.h"

namespace dbw {

inline int elem_bytes(int32_t dtype) { return dtype == DBW_F32 ? 4 : 2; }
inline bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// 16-byte (8-byte) vectors at addresses aligned to their elements only: global
// memory takes them, and the compiler emits one load or store.
typedef uint32_t lm_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t lm_u32x2 __attribute__((ext_vector_type(2)));
typedef lm_u32x4 lm_u32x4_any __attribute__((aligned(2)));
typedef lm_u32x2 lm_u32x2_any __attribute__((aligned(2)));
typedef float lm_f32x4 __attribute__((ext_vector_type(4)));
typedef float lm_f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ float lm_to_f32(float x) { return x; }
__device__ __forceinline__ float lm_to_f32(__bf16 x) { return static_cast<float>(x); }
__device__ __forceinline__ float lm_to_f32(_Float16 x) { return static_cast<float>(x); }

// ---------------------------------------------------------------------------
// offsets[i] of n + 1, taken into [0, T]
__device__ __forceinline__ int64_t lm_offset(const int32_t* offsets, int i, int64_t T) {
  const int64_t o = offsets[i];
  return o < 0 ? 0 : (o > T ? T : o);
}

// Inclusive sum over the 64 lanes of a wave.
__device__ __forceinline__ uint32_t lm_wave_scan(uint32_t v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t u = __shfl_up(v, d);
    if (lane >= d) v += u;
  }
  return v;
}

// ---------------------------------------------------------------------------
// Token loss.
struct TokenArgs {
  int n, C;
  int64_t T;
  int dtype;
  const int32_t* offsets;
  const void* Z;
  int64_t ld_Z;
  const int32_t* y;
  float scale;
  void* dZ;        // nullable
  int64_t ld_dZ;
  float* loss;     // [n]
  float* row_loss; // workspace [T]
  int32_t* counts; // workspace [n][parts]: live rows of a worker's part
  double* sums;    // workspace [n][parts]: sums of their losses
  int parts;       // parts of a worker's rows (set by the launch)
};
constexpr int kTokenParts = 64;
hipError_t launch_token_loss(const TokenArgs& a, hipStream_t s);

// ---------------------------------------------------------------------------
// AdamW.
constexpr int kAdamBlock = 256;    // values of one scale (8-bit states): a wave, four values a lane
constexpr int kAdamChunk = 1024;   // values of one tensor that a workgroup updates
constexpr int kAdamNormParts = 2048;

struct AdamTensor {
  float* w;
  const void* g;
  void* m;
  void* v;
  uint8_t* m_scale;
  uint8_t* v_scale;
  void* low;
  int64_t count;
  double lr_scale, decay;
};
struct AdamChunk {
  int32_t tensor;
  uint32_t index;  // chunk of the tensor
};
// Values of one step that all workgroups share, made by its first kernel.
struct AdamStep {
  int64_t t;
  float f, pre;     // factors of the gradients: f, behind pre = 1 or 2^-64
  float ibc2;       // 1 / sqrt(1 - beta2^t)
  double ibc1;      // 1 / (1 - beta1^t)
  uint32_t key;     // mix(mix(seed) + t)
  int32_t skip;     // the norm is not finite: leave everything
};
struct AdamArgs {
  const AdamTensor* tensors;
  const AdamChunk* chunks;
  int64_t nchunks;
  AdamStep* step;
  double* parts;    // [kAdamNormParts] sums of squares
  int bits, g_dtype, low_dtype;
  dbw_adamw_hyper h;
  float* norm;      // nullable
};
hipError_t launch_adamw(const AdamArgs& a, hipStream_t s);

// For dbw_set_adamw: the w at whose place the gradient buffer g [P] stands for
// all tensors of a plan; the failing tensor's number and reason in *why.
dbw_status adamw_place(const dbw_adamw* o, int device, const float* g, int64_t P, const float** w, std::string* why);
dbw_status adamw_check(const dbw_adamw_hyper& h, std::string* why);

// Rounding bits (see dbw_adamw_bits).
__host__ __device__ inline uint32_t adam_mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x9E3779B1u;
  x ^= x >> 15;
  x *= 0xB7E15163u;
  return x ^ (x >> 16);
}
__host__ __device__ inline uint32_t adam_index(int64_t index) {
  const uint64_t i = static_cast<uint64_t>(index);
  return static_cast<uint32_t>(i) * 0x6A09E667u + static_cast<uint32_t>(i >> 32) * 0xBB67AE85u;
}

// Sums over the 64 lanes of a wave, in every lane: four steps within 16 lanes,
// and the four 16s.
template <int CONTROL>
__device__ __forceinline__ uint32_t lm_moved(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CONTROL, 0xf, 0xf, true));
}
__device__ __forceinline__ uint32_t lm_lane(uint32_t v, int lane) {
  return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), lane));
}
__device__ __forceinline__ uint32_t lm_wave_sum(uint32_t v) {
  v += lm_moved<0xB1>(v);    // lanes 1, 0, 3, 2
  v += lm_moved<0x4E>(v);    // lanes 2, 3, 0, 1
  v += lm_moved<0x141>(v);   // halves of 16 lanes mirrored
  v += lm_moved<0x140>(v);   // 16 lanes mirrored
  return lm_lane(v, 0) + lm_lane(v, 16) + lm_lane(v, 32) + lm_lane(v, 48);
}
__device__ __forceinline__ float lm_wave_sum(float v) {
  const auto moved = [&](auto control) {
    return __builtin_bit_cast(float, lm_moved<decltype(control)::value>(__builtin_bit_cast(uint32_t, v)));
  };
  v += moved(std::integral_constant<int, 0xB1>{});
  v += moved(std::integral_constant<int, 0x4E>{});
  v += moved(std::integral_constant<int, 0x141>{});
  v += moved(std::integral_constant<int, 0x140>{});
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  return (__builtin_bit_cast(float, lm_lane(u, 0)) + __builtin_bit_cast(float, lm_lane(u, 16))) +
         (__builtin_bit_cast(float, lm_lane(u, 32)) + __builtin_bit_cast(float, lm_lane(u, 48)));
}

// ---------------------------------------------------------------------------
// Rows of ragged groups in chunks of `rows` rows: chunk number `slot` belongs
// to the group i with the largest (offsets[i] - offsets[0]) / rows + i that is
// not above it (a group has its first row's number of whole chunks, and one
// more for each group before it, in front of it, so that groups' slots never
// meet); T / rows + n slots hold all chunks, and some stay empty.  A whole wave
// looks at 64 groups at once.
struct LmChunk {
  int group;
  int32_t first;    // the chunk's first row
  int32_t start;    // the group's
  int32_t end;
  __device__ bool empty() const { return first >= end; }
};
__device__ __forceinline__ uint32_t lm_first_slot(const int32_t* offsets, int i, int64_t T, uint32_t o0, uint32_t rows) {
  const uint32_t o = static_cast<uint32_t>(lm_offset(offsets, i, T));
  return (o > o0 ? o - o0 : 0) / rows + i;
}
__device__ __forceinline__ LmChunk lm_chunk(const int32_t* offsets, int n, int64_t T, uint32_t rows, uint32_t slot,
                                            int lane) {
  const uint32_t o0 = static_cast<uint32_t>(lm_offset(offsets, 0, T));
  int lo = 0, count = n;
  while (count > 1) {
    const int step = (count + 63) / 64, at = lane * step;
    const bool below = at < count && lm_first_slot(offsets, lo + at, T, o0, rows) <= slot;
    const uint64_t past = __ballot(below);
    const int k = past ? 63 - __builtin_clzll(past) : 0;
    lo += k * step;
    count = count - k * step < step ? count - k * step : step;
  }
  LmChunk c;
  c.group = lo;
  const int64_t start = lm_offset(offsets, lo, T);
  const uint32_t first = lm_first_slot(offsets, lo, T, o0, rows);
  const int64_t row = start + static_cast<int64_t>(slot > first ? slot - first : 0) * rows;
  c.start = static_cast<int32_t>(start);
  c.end = static_cast<int32_t>(lm_offset(offsets, lo + 1, T));
  c.first = row < c.end ? static_cast<int32_t>(row) : c.end;
  c.group = __builtin_amdgcn_readfirstlane(c.group);
  c.start = __builtin_amdgcn_readfirstlane(c.start);
  c.end = __builtin_amdgcn_readfirstlane(c.end);
  c.first = __builtin_amdgcn_readfirstlane(c.first);
  return c;
}

// ---------------------------------------------------------------------------
// Activations: z sigmoid(s(z)) with s = 2 (a z + b z^3) or z, or simpler ones.
constexpr float kLog2E = 1.44269504088896341f;
constexpr float kGeluA = 0.797884560802865356f, kGeluB = 0.0356774081363001f;   // sqrt(2/pi), 0.044715 sqrt(2/pi)
__device__ __forceinline__ float lm_act(float z, int act) {
  if (act == DBW_ACT_RELU) return z < 0.f ? 0.f : z;   // (a NaN stays)
  if (act == DBW_ACT_NONE) return z;
  // exp(-s) as a power of two, with the factors joined
  const float s = act == DBW_ACT_GELU ? z * fmaf(-2.f * kLog2E * kGeluB, z * z, -2.f * kLog2E * kGeluA) : -kLog2E * z;
  return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(s));
}
// p + z p (1 - p) s'(z) with p = sigmoid(s): 1 - p as e / (1 + e), so that it keeps
// its digits where p is near 1 (1 - p by subtraction left 1e-5 of GELU's slope at
// 5).  Beyond the limits of z the slope is 0 or 1 to 2^-100, and e = exp(-s) not
// finite.
__device__ __forceinline__ float lm_act_slope(float z, int act) {
  if (act == DBW_ACT_RELU) return z > 0.f ? 1.f : (z <= 0.f ? 0.f : z);
  if (act == DBW_ACT_NONE) return 1.f;
  const bool gelu = act == DBW_ACT_GELU;
  const float most = gelu ? 10.f : 80.f;
  z = z > most ? most : (z < -most ? -most : z);   // (a NaN stays)
  const float s = gelu ? 2.f * z * fmaf(kGeluB * z, z, kGeluA) : z;
  const float ds = gelu ? 2.f * fmaf(3.f * kGeluB * z, z, kGeluA) : 1.f;
  const float e = __builtin_amdgcn_exp2f(-kLog2E * s), p = __builtin_amdgcn_rcpf(1.f + e);
  return fmaf(z * p * (e * p), ds, p);
}

// Where two waves share a SIMD, one of them goes first in everything, so that
// the other multiplies while it does not, and the other way around: waves that
// take turns stay in step, and the matrix cores wait for both at once.
__device__ __forceinline__ void lm_one_first() {
  if (__builtin_amdgcn_s_getreg(3 << 11 | 4) & 1) __builtin_amdgcn_s_setprio(2);   // by the wave's place in its SIMD
}

// ---------------------------------------------------------------------------
// Layer norm, the gradient of an activation with its bias, dropout.
struct NormArgs {
  int n, d;
  int64_t T;
  int dtype;
  const int32_t* offsets;
  const void* dY;       // gradient only
  int64_t ld_dY;
  const void* X;
  int64_t ld_X;
  const float* gamma;
  const float* beta;    // forward only, nullable
  float eps;
  void* out;            // Y or dX
  int64_t ld_out;
  float* dgamma;
  int64_t ld_dgamma;
  float* dbeta;         // nullable
  int64_t ld_dbeta;
  float* parts;         // workspace [2][parts_of_rows + n][d]: sums over pieces of the groups
  uint32_t rows, parts_of_rows;   // rows of a part (set by the launch)
};
constexpr int kNormMost = 16384;
int64_t norm_workspace(int n, int64_t T, int d);
hipError_t launch_layer_norm(const NormArgs& a, hipStream_t s);
hipError_t launch_layer_norm_grad(NormArgs a, hipStream_t s);

struct LinearGradArgs {
  int n, C;
  int64_t T;
  int dtype, act;
  const int32_t* offsets;
  const void* dY;
  int64_t ld_dY;
  const void* Z;        // nullable: no activation
  int64_t ld_Z;
  void* dZ;             // nullable
  int64_t ld_dZ;
  float* dbias;         // nullable
  int64_t ld_dbias;
  float* parts;         // workspace [parts of the rows + n][C]
  uint32_t rows;
};
int64_t linear_grad_workspace(int n, int64_t T, int C);
hipError_t launch_linear_grad(LinearGradArgs a, hipStream_t s);

struct DropoutArgs {
  int n, d;
  int64_t T;
  int dtype;
  const int32_t* offsets;
  const void* X;
  int64_t ld_X;
  const void* R;        // nullable
  int64_t ld_R;
  void* Y;
  int64_t ld_Y;
  uint32_t cut;         // dropped below
  float scale;
  uint64_t seed;
  const int64_t* step;  // nullable
};
hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s);

// Philox4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", 2011).
__host__ __device__ inline void lm_philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p = static_cast<uint64_t>(0xD2511F53u) * c[0], q = static_cast<uint64_t>(0xCD9E8D57u) * c[2];
    c[0] = static_cast<uint32_t>(q >> 32) ^ c[1] ^ k0;
    c[1] = static_cast<uint32_t>(q);
    c[2] = static_cast<uint32_t>(p >> 32) ^ c[3] ^ k1;
    c[3] = static_cast<uint32_t>(p);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

// ---------------------------------------------------------------------------
// Attention.
struct HeadRows {
  char* p;
  int64_t token, head;  // elements
};
struct AttentionArgs {
  int n, heads, kv_heads, D;
  int64_t T;
  int dtype;
  float scale;
  const int32_t* offsets;
  HeadRows Q, K, V, O, dO, dQ, dK, dV;
  float* lse;           // [heads][T], nullable in the forward pass
  // workspace [3][heads][T]: dO . O; lse log2(e) and 0, or, where that is large for one
  // of 128 rows, the logarithm (of 2) of sum exp(S - maximum) and the maximum of Q . K
  float* delta;
  float* sums;          // workspace [parts][2][T][kv_heads][D] (parts > 1)
  int parts;            // workgroups that share the queries of a tile of keys
  uint32_t slots;       // tiles of a head's queries or keys (set by the launch)
};
int attention_parts(int n, int64_t T, int heads, int kv_heads);
constexpr int kAttentionKeys = 64;   // the fewest rows of a workgroup (512 threads)
hipError_t launch_attention(AttentionArgs a, hipStream_t s);
hipError_t launch_attention_grad(AttentionArgs a, hipStream_t s);

// ---------------------------------------------------------------------------
// Grouped products.
struct GroupPlan {
  int variant = 0;        // GroupVariant
  int splits = 1;         // parts of the sum, each with its own partial output
  int64_t row_tiles = 0;  // most row tiles (FORWARD, INPUT_GRAD) or tiles of d (WEIGHT_GRAD)
  int64_t col_tiles = 0;
  int64_t part = 0;       // floats of one partial output (splits > 1)
  int64_t tiles = 0;      // output tiles, with rows spread evenly over the groups
  int64_t blocks = 0;     // workgroups
};
GroupPlan group_plan(const dbw_group_shape& p);
// epilogue: nullptr, or that of a FORWARD product
hipError_t launch_group(const dbw_group_shape& p, GroupPlan plan, const int32_t* offsets, const void* a,
                        const void* b, void* out, float* workspace, const dbw_linear_epilogue* epilogue, hipStream_t s);

}  // namespace dbw
