// Matrix-core operands of a work item of step attention over an 8-bit cache: a whole page of 128 keys, 16-byte loads of 16 codes that
// become two bf16 operands of v_mfma_f32_16x16x32_bf16, exactly (e4m3.h).
//
// Products: a query in bf16 is one operand, in fp32 three (its upper 8 bits, the next 8, the rest: truncated, so that no part exceeds
// bf16's range, and exact); probabilities enter as two bf16 terms beside bf16 queries, as in decode_shape.h, and as their three parts
// beside fp32 ones.
#pragma once

#include "decode_shape.h"
#include "e4m3.h"

namespace actqkv {

// The upper halves of two fp32 values, packed, and what is left of the values.
__device__ __forceinline__ uint32_t upper_halves(float& x0, float& x1) {
  const uint32_t a = __float_as_uint(x0) & 0xffff0000u, b = __float_as_uint(x1) & 0xffff0000u;
  x0 -= __uint_as_float(a), x1 -= __uint_as_float(b);
  return a >> 16 | b;
}

// MFMA row r of sub-tile j = 2 st + h is key 64 (st / 2) + 16 (r / 4) + 8 (st % 2) + 4 h + r % 4: lane quarter kq ends up with keys
// 16 kq + 8 (st % 2) .. + 7 of the 64 in steps st, which a 16-byte load of values brings for two steps.  Channels likewise: load c
// of a key is channels 64 c + 16 kq .. + 15, the operands of steps 2 c and 2 c + 1.
template <typename T, int D>
struct Step8Shape {
  typedef uint8_t elem;
  static constexpr bool kScaled = true;
  static constexpr int kParts = sizeof(T) == 2 ? 1 : 3;
  static constexpr int kKeys = kBlock, kSubs = kKeys / 16, kSteps = kKeys / 32;
  static constexpr int kC = D / 64, kQ = D / 32, kQRegs = kQ * kParts;
  static constexpr int kK = kSubs * kC, kV = (D / 16) * (kKeys / 64);
  __device__ static __forceinline__ int key_of(int j, int i, int kq) {
    return 64 * (j >> 2) + 16 * kq + 8 * ((j >> 1) & 1) + 4 * (j & 1) + i;
  }
  __device__ static __forceinline__ int k_lane(int n, int kq) { return (16 * (n >> 2) + (n & 3)) * D + 16 * kq; }
  __device__ static __forceinline__ int k_off(int l) {
    const int j = l / kC;
    return (64 * (j >> 2) + 8 * ((j >> 1) & 1) + 4 * (j & 1)) * D + 64 * (l % kC);
  }
  __device__ static __forceinline__ int v_lane(int n, int kq) { return n * kBlock + 16 * kq; }
  __device__ static __forceinline__ int v_off(int l) { return 16 * (l >> 1) * kBlock + 64 * (l & 1); }
  __device__ static __forceinline__ int v_key(int l, int kq) { return 64 * (l & 1) + 16 * kq; }
  __device__ static __forceinline__ void clear_behind(u32x4& va, int key, int end) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int there = min(max(end - key - 4 * i, 0), 4);         // bytes of the word
      va[i] &= there == 4 ? ~0u : (1u << (8 * there)) - 1u;
    }
  }
  __device__ static __forceinline__ void load_q(const T* q, int kq, u32x4 (&qb)[kQRegs]) {
#pragma unroll
    for (int ks = 0; ks < kQ; ++ks) {
      const T* from = q + 64 * (ks >> 1) + 16 * kq + 8 * (ks & 1);
      if constexpr (kParts == 1) {
        qb[ks] = *reinterpret_cast<const u32x4*>(from);
      } else {
        f32x4 x[2] = {*reinterpret_cast<const f32x4*>(from), *reinterpret_cast<const f32x4*>(from + 4)};
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x0 = x[i >> 1][2 * (i & 1)], x1 = x[i >> 1][2 * (i & 1) + 1];
            qb[part * kQ + ks][i] = upper_halves(x0, x1);
            x[i >> 1][2 * (i & 1)] = x0, x[i >> 1][2 * (i & 1) + 1] = x1;
          }
      }
    }
  }
  __device__ static __forceinline__ bf16x8 operand(const u32x4& codes, int half, float scale) {
    return dc_as_bf16x8(e4m3_bf16x8(codes[2 * half], codes[2 * half + 1], scale));
  }
  __device__ static __forceinline__ void scores(const u32x4 (&ka)[kK], const u32x4 (&qb)[kQRegs], float scale, f32x4 (&sc)[kSubs]) {
#pragma unroll
    for (int ks = 0; ks < kQ; ++ks)
#pragma unroll
      for (int j = 0; j < kSubs; ++j) {
        const bf16x8 k = operand(ka[j * kC + (ks >> 1)], ks & 1, scale);
#pragma unroll
        for (int part = kParts - 1; part >= 0; --part)
          sc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, dc_as_bf16x8(qb[part * kQ + ks]), sc[j], 0, 0, 0);
      }
  }
  __device__ static __forceinline__ void values(const u32x4 (&va)[kV], const f32x4 (&sc)[kSubs], float scale, f32x4 (&acc)[D / 16]) {
    typedef __attribute__((ext_vector_type(8))) float f32x8;
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
      f32x8 left = {sc[2 * st][0], sc[2 * st][1], sc[2 * st][2], sc[2 * st][3],
                    sc[2 * st + 1][0], sc[2 * st + 1][1], sc[2 * st + 1][2], sc[2 * st + 1][3]};
      constexpr int kTerms = kParts == 1 ? 2 : 3;
      bf16x8 p[kTerms];
#pragma unroll
      for (int i = 0; i < kTerms; ++i) {
        p[i] = __builtin_convertvector(left, bf16x8);
        left -= __builtin_convertvector(p[i], f32x8);
      }
#pragma unroll
      for (int dg = 0; dg < D / 16; ++dg) {
        const bf16x8 v = operand(va[2 * dg + (st >> 1)], st & 1, scale);
#pragma unroll
        for (int i = kTerms - 1; i >= 0; --i) acc[dg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[i], acc[dg], 0, 0, 0);
      }
    }
  }
};

}  // namespace actqkv
