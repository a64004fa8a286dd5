// The pieces of a query tile of the paged attention, and their merge by a second launch.
//
// A piece is, per wavefront that holds output: 16-byte slots of it, unnormalised fp32, in the order the registers hold it (slot 4 j + k
// is registers 4 k .. 4 k + 3 of 32-channel group j), 64 lanes each, then (maximum, sum) of the lane's row.  A piece that had no pages
// is (-infinity, 0) alone.  The workgroup that finishes last could merge as well, but it reads the others' results past
// the L2s, 31 us for 8 pieces of 128 rows; the launch takes 4 to 5.
#pragma once

#include "paged.h"

namespace actqkv {

// kRowGroups: sets of 32 rows of a query tile; kMine: 32-channel groups of a wavefront; kQuarters: wavefronts that share a row set.
template <int kRowGroups, int kMine, int kQuarters>
struct PagedPiece {
  static constexpr int kWaves = kRowGroups * kQuarters, kSlots = 4 * kMine;
  static constexpr int kWords = kSlots * 64 + 32;      // 16-byte words of a wavefront
  static __host__ __device__ constexpr size_t bytes() { return size_t(kWaves) * kWords * 16; }
  static __device__ __forceinline__ u32x4* at(void* part, int item, int splits, int split, int wave) {
    return static_cast<u32x4*>(part) + ((size_t(item) * splits + split) * kWaves + wave) * kWords;
  }
  static __device__ __forceinline__ void store(u32x4* to, const f32x16 (&o)[kMine], float m, float l, int lane) {
#pragma unroll
    for (int k = 0; k < kSlots; ++k)
      to[k * 64 + lane] = u32x4{__float_as_uint(o[k / 4][4 * (k % 4)]), __float_as_uint(o[k / 4][4 * (k % 4) + 1]),
                                __float_as_uint(o[k / 4][4 * (k % 4) + 2]), __float_as_uint(o[k / 4][4 * (k % 4) + 3])};
    store_none(to, m, l, lane);
  }
  static __device__ __forceinline__ void store_none(u32x4* to, float m, float l, int lane) {
    reinterpret_cast<f32x2*>(to + kSlots * 64)[lane] = f32x2{m, l};
  }
};

struct PagedMerge {
  PagedAttn a;
  int tiles, splits;
  void* part;
};
// A wavefront merges kTake slots of the 32 rows of a wavefront of the attention; grid (tiles * Hk, kWaves * kSlots / kTake / 4).
constexpr int kPmThreads = 256, kPmTake = 2;
template <typename T, int D, int kRowGroups, int kMine, int kQuarters>
__device__ __forceinline__ void merge_body(const PagedMerge& c) {
  typedef PagedPiece<kRowGroups, kMine, kQuarters> Piece;
  constexpr int kParts = Piece::kSlots / kPmTake, kBatch = 8;
  const PagedAttn& p = c.a;
  const int lane = threadIdx.x & 63, n = lane & 31, half = lane >> 5;
  const int hk = blockIdx.x % p.n_kv_heads, tile = blockIdx.x / p.n_kv_heads, group = p.n_q_heads / p.n_kv_heads;
  const int unit = blockIdx.y * (kPmThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= Piece::kWaves * kParts) return;
  const int wave = unit / kParts, part = unit % kParts;
  int s = 0, qtile = 0;
  if (!paged_find_tile(p.t, tile, group, 32 * kRowGroups, s, qtile)) return;
  const PagedSeq seq = paged_seq(p.t, s);
  float m = -INFINITY, l = 0.f;
  f32x4 o[kPmTake];
#pragma unroll
  for (int k = 0; k < kPmTake; ++k) o[k] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int i0 = 0; i0 < c.splits; i0 += kBatch) {
    f32x2 ml[kBatch];
    u32x4 raw[kBatch][kPmTake];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {             // all loads first: they overlap
      const u32x4* from = Piece::at(c.part, tile * p.n_kv_heads + hk, c.splits, min(i0 + i, c.splits - 1), wave);
      ml[i] = reinterpret_cast<const f32x2*>(from + Piece::kSlots * 64)[lane];
#pragma unroll
      for (int k = 0; k < kPmTake; ++k) raw[i][k] = from[(part * kPmTake + k) * 64 + lane];
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (i0 + i < c.splits && ml[i].y > 0.f) {    // (of a piece without pages there is no output)
        const float m_new = fmaxf(m, ml[i].x), a = __builtin_amdgcn_exp2f(m - m_new), b = __builtin_amdgcn_exp2f(ml[i].x - m_new);
        m = m_new;
        l = l * a + ml[i].y * b;
#pragma unroll
        for (int k = 0; k < kPmTake; ++k)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[k][r] = o[k][r] * a + __uint_as_float(raw[i][k][r]) * b;
      }
    }
  }
  const int frow = qtile * (32 * kRowGroups) + (wave % kRowGroups) * 32 + n;
  if (frow >= seq.m * group) return;
  const int i_row = frow / group, head = hk * group + (frow - i_row * group);
  const size_t at = size_t(seq.row0 + i_row) * p.n_q_heads + head;
  const float inv = l > 0.f ? 1.f / l : 0.f;
  const int db0 = wave / kRowGroups * kMine;
#pragma unroll
  for (int k = 0; k < kPmTake; ++k) {
    const int slot = part * kPmTake + k;
    T* to = static_cast<T*>(p.out) + at * D + (db0 + slot / 4) * 32 + 8 * (slot % 4) + 4 * half;
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16x2(o[k][0] * inv, o[k][1] * inv), pack_bf16x2(o[k][2] * inv, o[k][3] * inv)};
    else
      *reinterpret_cast<f32x4*>(to) = o[k] * inv;
  }
  if (p.lse != nullptr && half == 0 && db0 == 0 && part == 0) p.lse[at] = (m + log2f(l)) * kLn2;
}
template <typename T, int D, int kRowGroups, int kMine, int kQuarters>
__global__ __launch_bounds__(kPmThreads) void paged_merge_kernel(PagedMerge c) {
  merge_body<T, D, kRowGroups, kMine, kQuarters>(c);
}
template <typename T, int D, int kRowGroups, int kMine, int kQuarters>
inline void launch_paged_merge(const PagedMerge& c, hipStream_t stream) {
  typedef PagedPiece<kRowGroups, kMine, kQuarters> Piece;
  constexpr int kUnits = Piece::kWaves * (Piece::kSlots / kPmTake), kPer = kPmThreads / 64;
  hipLaunchKernelGGL((paged_merge_kernel<T, D, kRowGroups, kMine, kQuarters>),
                     dim3(unsigned(c.tiles) * c.a.n_kv_heads, (kUnits + kPer - 1) / kPer), dim3(kPmThreads), 0, stream, c);
}

}  // namespace actqkv
