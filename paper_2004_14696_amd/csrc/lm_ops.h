// Internal declarations of the operators for language models: grouped
// products, token loss, AdamW.  Not part of the C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "dbw.h"

namespace dbw {

inline int elem_bytes(int32_t dtype) { return dtype == DBW_F32 ? 4 : 2; }

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
hipError_t launch_group(const dbw_group_shape& p, GroupPlan plan, const int32_t* offsets, const void* a,
                        const void* b, void* out, float* workspace, hipStream_t s);

}  // namespace dbw
