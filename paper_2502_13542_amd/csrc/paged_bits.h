// Which pages a row sees, as bits: lists of selected pages in the form that attention of many rows takes them in.
#pragma once

#include "paged.h"

namespace actqkv {

constexpr int kMostBitWords = 256;                 // 8192 pages
struct PagedBits {
  const uint32_t* bits;                            // [n_rows][Hk][words]
  int words;
  __device__ __forceinline__ const uint32_t* of(int row, int hk, int n_kv_heads) const {
    return bits + (size_t(row) * n_kv_heads + hk) * words;
  }
};
// The pages that any of n rows sees, in LDS.
template <int kThreads>
__device__ __forceinline__ void any_chosen(const PagedBits& b, int row0, int n, int hk, int n_kv_heads, uint32_t* any) {
  for (int i = threadIdx.x; i < b.words; i += kThreads) any[i] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n * b.words; i += kThreads) {
    const uint32_t v = b.of(row0 + i / b.words, hk, n_kv_heads)[i % b.words];
    if (v != 0) atomicOr(any + i % b.words, v);
  }
  __syncthreads();
}
// The first of them from page t on, or `end`; the same in all lanes.
__device__ __forceinline__ int next_chosen(const uint32_t* any, int t, int end) {
  while (t < end) {
    const uint32_t rest = __builtin_amdgcn_readfirstlane(any[t >> 5]) >> (t & 31);
    if (rest != 0) return min(t + __builtin_ctz(rest), end);
    t = (t | 31) + 1;
  }
  return end;
}

}  // namespace actqkv
