// fp32 products on the 16-bit matrix cores: a value as three bf16 parts, a product as six of theirs (attn_prefill_f32.hip has
// the arithmetic).
#pragma once

#include "common.h"

namespace actqkv {

constexpr float kFfMax = 3.3895314e38f;           // the largest bf16: what is larger has no parts

// Two fp32 values -> their three parts, packed.  What is left of a value after a part is exact.
__device__ __forceinline__ void ff_split(float x0, float x1, uint32_t (&part)[3]) {
  part[0] = pack_bf16x2(x0, x1);
  x0 -= bf16_lo(part[0]), x1 -= bf16_hi(part[0]);
  part[1] = pack_bf16x2(x0, x1);
  x0 -= bf16_lo(part[1]), x1 -= bf16_hi(part[1]);
  part[2] = pack_bf16x2(x0, x1);
}
// The same of the values times scale, to 2^-26 of them.
__device__ __forceinline__ void ff_split_scaled(float x0, float x1, float scale, uint32_t (&part)[3]) {
  part[0] = pack_bf16x2(x0 * scale, x1 * scale);
  x0 = fmaf(x0, scale, -bf16_lo(part[0])), x1 = fmaf(x1, scale, -bf16_hi(part[0]));
  part[1] = pack_bf16x2(x0, x1);
  x0 -= bf16_lo(part[1]), x1 -= bf16_hi(part[1]);
  part[2] = pack_bf16x2(x0, x1);
}
__device__ __forceinline__ bf16x8 ff_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }
__device__ __forceinline__ f32x16 ff_mfma(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// The six products of a step, small ones first: part kFfOf[i][0] of one factor, kFfOf[i][1] of the other.
constexpr int kFfProducts = 6;
constexpr int kFfOf[kFfProducts][2] = {{2, 0}, {1, 1}, {0, 2}, {1, 0}, {0, 1}, {0, 0}};

}  // namespace actqkv
