// Dropout with the residual's addition; the mask is drawn again wherever it is
// needed, from a counter: eight values of a row take one Philox4x32-10 block, 16
// bits each.
//
// Bound by memory: 16384 x 4096 bf16 with a residual 73 us, 5.5 TB/s.  The 20
// products of 32 by 32 bits of a block, 16 cycles each, are a quarter of the time that
// memory takes for a wave's 512 values; with 32 bits a value they would be half.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "lm_ops.h"

namespace dbw {
namespace {

template <typename E>
struct Eight {
  static constexpr int WORDS = sizeof(E) * 2;   // of 32 bits
  typedef E V __attribute__((ext_vector_type(8)));
  typedef uint32_t U __attribute__((ext_vector_type(WORDS)));
  E x[8];
  __device__ __forceinline__ void load(const E* p, int left) {
    if (left >= 8) {
      lm_u32x4 w[WORDS / 4];
#pragma unroll
      for (int i = 0; i < WORDS / 4; ++i) w[i] = *reinterpret_cast<const lm_u32x4_any*>(p + i * (16 / sizeof(E)));
      __builtin_memcpy(x, w, sizeof x);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = j < left ? p[j] : static_cast<E>(0.f);
    }
  }
  __device__ __forceinline__ void store(E* p, int left) const {
    if (left >= 8) {
      lm_u32x4 w[WORDS / 4];
      __builtin_memcpy(w, x, sizeof x);
#pragma unroll
      for (int i = 0; i < WORDS / 4; ++i) *reinterpret_cast<lm_u32x4_any*>(p + i * (16 / sizeof(E))) = w[i];
    } else {
#pragma unroll
      for (int j = 0; j < 7; ++j)
        if (j < left) p[j] = x[j];
    }
  }
};

template <typename E>
__global__ __launch_bounds__(256) void k_dropout(DropoutArgs a) {
  const uint32_t blocks = (a.d + 7) / 8;
  const int64_t first = lm_offset(a.offsets, 0, a.T), end = lm_offset(a.offsets, a.n, a.T);
  const uint64_t step = a.step ? static_cast<uint64_t>(*a.step) : 0;
  const int64_t all = (end - first) * blocks, stride = static_cast<int64_t>(gridDim.x) * 256;
  const E* X = static_cast<const E*>(a.X);
  const E* R = static_cast<const E*>(a.R);
  E* Y = static_cast<E*>(a.Y);
  int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  int64_t t = first + i / blocks;
  uint32_t b = static_cast<uint32_t>(i % blocks);
  const int64_t more_t = stride / blocks;
  const uint32_t more_b = static_cast<uint32_t>(stride % blocks);
  for (; i < all; i += stride) {
    const int c = static_cast<int>(b) * 8, left = a.d - c;
    Eight<E> x, r;
    x.load(X + t * a.ld_X + c, left);
    if (R) r.load(R + t * a.ld_R + c, left);
    uint32_t u[4] = {b, static_cast<uint32_t>(t), static_cast<uint32_t>(step), static_cast<uint32_t>(step >> 32)};
    lm_philox(u, static_cast<uint32_t>(a.seed), static_cast<uint32_t>(a.seed >> 32));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t bits = j % 2 ? u[j / 2] >> 16 : u[j / 2] & 0xffffu;
      float y = bits >= a.cut ? lm_to_f32(x.x[j]) * a.scale : 0.f;
      if (R) y += lm_to_f32(r.x[j]);
      x.x[j] = static_cast<E>(y);
    }
    x.store(Y + t * a.ld_Y + c, left);
    t += more_t;
    b += more_b;
    if (b >= blocks) {
      b -= blocks;
      ++t;
    }
  }
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s) {
  if (a.T == 0) return hipSuccess;
  const int64_t all = a.T * ((a.d + 7) / 8);
  const uint32_t grid = static_cast<uint32_t>(std::min<int64_t>((all + 255) / 256, 8192));
  if (a.dtype == DBW_F32) k_dropout<float><<<grid, 256, 0, s>>>(a);
  else if (a.dtype == DBW_BF16) k_dropout<__bf16><<<grid, 256, 0, s>>>(a);
  else k_dropout<_Float16><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace dbw
