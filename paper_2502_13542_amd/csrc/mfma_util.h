// Small helpers of the kernels on the 16-bit matrix cores.
#pragma once

#include "common.h"

namespace actqkv {

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

// 8 fp32 -> 8 bf16 (round to nearest even), packed as an MFMA operand
__device__ __forceinline__ bf16x8 pack8(float a0, float a1, float a2, float a3, float a4, float a5,
                                        float a6, float a7) {
  typedef __attribute__((ext_vector_type(8))) float f32x8;
  f32x8 v = {a0, a1, a2, a3, a4, a5, a6, a7};
  return __builtin_convertvector(v, bf16x8);
}

// A pointer that is the same in all lanes, pinned to scalar registers (so that adding a
// 32-bit lane offset to it becomes the scalar-base addressing mode of the load).
__device__ __forceinline__ const char* uniform_ptr(const char* ptr) {
  const uint64_t v = reinterpret_cast<uint64_t>(ptr);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(v));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(uint32_t(v >> 32));
  return reinterpret_cast<const char*>((uint64_t(hi) << 32) | lo);
}

// MFMA row -> key row inside a 32-key group: swap bits 2 and 3.
__device__ __forceinline__ int perm_row(int i) {
  return (i & ~12) | ((i & 4) << 1) | ((i & 8) >> 1);
}

}  // namespace actqkv
