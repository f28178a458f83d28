// What the kernels on the matrix cores share: loads straight into LDS, the wait
// for them, pairs of 16-bit values.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dbw_buffer.h"

namespace dbw {

// 16 bytes a lane from r + off + more (the same for all lanes) to the wave's 1 KiB
// at `to`.
__device__ __forceinline__ void load_lds(__amdgpu_buffer_rsrc_t r, char* to, uint32_t off, uint32_t more = 0) {
  typedef __attribute__((address_space(3))) void* P;
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (P)to, 16, off, static_cast<int>(more), 0, 0);
}

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

}  // namespace dbw
