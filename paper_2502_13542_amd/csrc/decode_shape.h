// The two matrix-core forms of a work item of decode attention, shared by the kernels over the blocked and the paged cache.
#pragma once

#include "common.h"

namespace actqkv {

__device__ __forceinline__ bf16x8 dc_as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

// The two matrix-core forms of an item.  kSubs accumulators of 16 keys x 16 heads hold the scores;
// key_of says which key of the item register i of accumulator j is in lane quarter kq.  kK and kV
// count the 16-byte loads of a lane for the item's keys and values, kQ those of its query.
template <typename T, int D> struct DcShape;
// bf16, v_mfma_f32_16x16x32_bf16.  MFMA row r of sub-tile h of 32-key step st is key
// 32*st + 8*(r/4) + 4*h + r%4, so that lane quarter kq ends up with keys 32*st + 8*kq + 4*h + i in
// register i: 8 consecutive keys per 32-key step, which is the B operand of the second product.
template <int D>
struct DcShape<uint16_t, D> {
  static constexpr int kKeys = 64;                 // keys per work item (half a block)
  static constexpr int kSubs = kKeys / 16, kSteps = kKeys / 32;
  static constexpr int kQ = D / 32, kK = kSubs * kQ, kV = (D / 16) * kSteps;
  __device__ static __forceinline__ int key_of(int j, int i, int kq) { return 32 * (j >> 1) + 8 * kq + 4 * (j & 1) + i; }
  // element offsets of a lane's operands from the item's first key (K rows) / first key column (V^T rows)
  __device__ static __forceinline__ int k_lane(int n, int kq) { return (8 * (n >> 2) + (n & 3)) * D + 8 * kq; }
  __device__ static __forceinline__ int k_off(int l) { return (32 * (l / (2 * kQ)) + 4 * ((l / kQ) & 1)) * D + (l % kQ) * 32; }
  __device__ static __forceinline__ int v_lane(int n, int kq) { return n * kBlock + 8 * kq; }
  __device__ static __forceinline__ int v_off(int l) { return 16 * (l / kSteps) * kBlock + 32 * (l % kSteps); }
  __device__ static __forceinline__ int q_lane(int kq) { return 8 * kq; }
  // first key of the item in a lane's l-th operand of the values, and that operand with what lies from key `end` on put to zero
  __device__ static __forceinline__ int v_key(int l, int kq) { return 32 * (l % kSteps) + 8 * kq; }
  __device__ static __forceinline__ void clear_behind(u32x4& va, int key, int end) {
#pragma unroll
    for (int i = 0; i < 4; ++i) va[i] &= (key + 2 * i < end ? 0xffffu : 0u) | (key + 2 * i + 1 < end ? 0xffff0000u : 0u);
  }
  static constexpr int kQStep = 32;
  __device__ static __forceinline__ void scores(const u32x4 (&ka)[kK], const u32x4 (&qb)[kQ], f32x4 (&sc)[kSubs]) {
#pragma unroll
    for (int ks = 0; ks < kQ; ++ks)      // the sub-tiles take turns: no MFMA waits for the one before it
#pragma unroll
      for (int j = 0; j < kSubs; ++j)
        sc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(dc_as_bf16x8(ka[j * kQ + ks]), dc_as_bf16x8(qb[ks]), sc[j], 0, 0, 0);
  }
  __device__ static __forceinline__ void values(const u32x4 (&va)[kV], const f32x4 (&sc)[kSubs], f32x4 (&acc)[D / 16]) {
    // The probabilities enter as two bf16 terms, the rounded value and what the rounding left, which keeps 16 of
    // their bits.  With one term the error grows with the keys a wavefront walks (a row's largest probability so far
    // is exactly 1, and fewer wavefronts have fewer of them).  Relative error against 64 bits, mean of 8 inputs, 48
    // sequences with 28 query and 4 KV heads of 128 channels: one term 1.768e-3 in two workgroups per pair, 1.791e-3
    // in one, two terms 1.676e-3; with 64 channels (8 query, 2 KV heads) one term 1.835e-3, two 1.727e-3, as
    // with fp32 probabilities.  A launch is bound by its bytes: a step of 16 sequences takes 186 us with two terms
    // and 188 with one, of 48 sequences 138 with both.
    typedef __attribute__((ext_vector_type(8))) float f32x8;
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
      f32x8 pf = {sc[2 * st][0], sc[2 * st][1], sc[2 * st][2], sc[2 * st][3],
                  sc[2 * st + 1][0], sc[2 * st + 1][1], sc[2 * st + 1][2], sc[2 * st + 1][3]};
      const bf16x8 pb = __builtin_convertvector(pf, bf16x8);
#pragma unroll
      for (int dg = 0; dg < D / 16; ++dg)
        acc[dg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(dc_as_bf16x8(va[dg * kSteps + st]), pb, acc[dg], 0, 0, 0);
      const bf16x8 pl = __builtin_convertvector(pf - __builtin_convertvector(pb, f32x8), bf16x8);
#pragma unroll
      for (int dg = 0; dg < D / 16; ++dg)
        acc[dg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(dc_as_bf16x8(va[dg * kSteps + st]), pl, acc[dg], 0, 0, 0);
    }
  }
};
// fp32, v_mfma_f32_16x16x4_f32 (fp32 products and sums throughout): the 16 channels of a step are
// dealt to the lane quarters four at a time, so that a lane's operand is a 16-byte load; register i
// of accumulator j is key 16*j + 4*kq + i, and the four MFMAs of the second product take the keys
// 4*kq + i, i = 0 .. 3, of every quarter: the scores are its B operand as they are.
template <int D>
struct DcShape<float, D> {
  static constexpr int kKeys = 4096 / D;           // 16 KB of keys and 16 KB of values, as for bf16 with D = 128
  static constexpr int kSubs = kKeys / 16;
  static constexpr int kQ = D / 16, kK = kSubs * kQ, kV = (D / 16) * kSubs;
  __device__ static __forceinline__ int key_of(int j, int i, int kq) { return 16 * j + 4 * kq + i; }
  __device__ static __forceinline__ int k_lane(int n, int kq) { return n * D + 4 * kq; }
  __device__ static __forceinline__ int k_off(int l) { return 16 * (l / kQ) * D + (l % kQ) * 16; }
  __device__ static __forceinline__ int v_lane(int n, int kq) { return n * kBlock + 4 * kq; }
  __device__ static __forceinline__ int v_off(int l) { return 16 * (l / kSubs) * kBlock + 16 * (l % kSubs); }
  __device__ static __forceinline__ int q_lane(int kq) { return 4 * kq; }
  __device__ static __forceinline__ int v_key(int l, int kq) { return 16 * (l % kSubs) + 4 * kq; }
  __device__ static __forceinline__ void clear_behind(u32x4& va, int key, int end) {
#pragma unroll
    for (int i = 0; i < 4; ++i) va[i] = key + i < end ? va[i] : 0u;
  }
  static constexpr int kQStep = 16;
  __device__ static __forceinline__ void scores(const u32x4 (&ka)[kK], const u32x4 (&qb)[kQ], f32x4 (&sc)[kSubs]) {
#pragma unroll
    for (int ks = 0; ks < kQ; ++ks)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < kSubs; ++j)
          sc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(ka[j * kQ + ks][i]), __uint_as_float(qb[ks][i]), sc[j], 0, 0, 0);
  }
  __device__ static __forceinline__ void values(const u32x4 (&va)[kV], const f32x4 (&sc)[kSubs], f32x4 (&acc)[D / 16]) {
#pragma unroll
    for (int j = 0; j < kSubs; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int dg = 0; dg < D / 16; ++dg)
          acc[dg] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(va[dg * kSubs + j][i]), sc[j][i], acc[dg], 0, 0, 0);
  }
};

}  // namespace actqkv
