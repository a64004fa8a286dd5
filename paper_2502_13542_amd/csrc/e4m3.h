// Values in 8 bits: e4m3 codes (a sign, 4 bits of exponent, 3 of the significand; the largest 448, the least 2^-9, no infinity) times a power of two
// that is shared by a KV head's tokens of a page, keys and values apart.
//
// A power of two costs nothing: codes keep their 4 significant bits whatever the scale is, values are exact in bf16 (the
// conversion instruction multiplies by it), and where a scale grows, codes move without a rounding as long as they stay above 2^-6.
#pragma once

#include "common.h"

namespace actqkv {

constexpr int kLeastE4m3 = -100, kMostE4m3 = 120;        // exponents of the scale (2^120 * 448 is above the largest fp32)

__device__ __forceinline__ float pow2f(int e) { return __uint_as_float(uint32_t(e + 127) << 23); }
// Of a scale in memory: the power of two alone, whatever it holds.
__device__ __forceinline__ int e4m3_exponent(float scale) {
  return min(max(int(__float_as_uint(scale) >> 23 & 255u) - 127, kLeastE4m3), kMostE4m3);
}
// The least e with most <= 448 * 2^e = 1.75 * 2^(e + 8); most is finite and not negative.
__device__ __forceinline__ int e4m3_exponent_for(float most) {
  const uint32_t bits = __float_as_uint(most);
  return max(int(bits >> 23) - 127 - 8 + int((bits & 0x7fffffu) > 0x600000u), kLeastE4m3);
}
// The largest value that a scale 2^e is the least for (448 2^e, but of the largest e what fp32 has).
__device__ __forceinline__ float e4m3_most(int e) { return e < kMostE4m3 ? 1.75f * pow2f(e + 8) : __uint_as_float(0x7f7fffffu); }
__device__ __forceinline__ uint32_t e4m3_pack(float x0, float x1, float x2, float x3) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x0, x1, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(x2, x3, lo, true);
}
// Four codes times a factor, as codes again.
__device__ __forceinline__ uint32_t e4m3_again(uint32_t codes, float by) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
  return e4m3_pack(lo[0] * by, lo[1] * by, hi[0] * by, hi[1] * by);
}
// The largest absolute value but for infinities and NaN.
__device__ __forceinline__ float largest(float most, float x) {
  const float a = fabsf(x);
  return a < INFINITY ? fmaxf(most, a) : most;
}
// Eight codes times their scale as eight bf16, exactly.
__device__ __forceinline__ u32x4 e4m3_bf16x8(uint32_t lo, uint32_t hi, float scale) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true))};
}

}  // namespace actqkv
