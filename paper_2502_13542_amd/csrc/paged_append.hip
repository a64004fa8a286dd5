// Keys and values of a ragged batch's new tokens into their pages (the paged form of Sec. 3.1, Eq. (4)).
//
// A workgroup takes half of the channels of the new tokens of one (sequence, KV head) that fall into one page: the keys go as
// they are, the values through LDS, two neighbouring tokens a word, so that a channel's row of the page is written in 16-byte
// stores where eight (fp32: four) neighbouring tokens are new.  All loads of a thread are in flight before the first store.
// Bound by HBM, a step by its launch.  32 query, 8 KV heads of 128, bf16: a token of each of 64 sequences 5.4 to 5.6 us, 15.4k tokens of
// 16 sequences, 126 MB in and out, 35 to 36 us = 3.6 TB/s; a plain copy of as many bytes takes 26: here all is one round of
// workgroups, whose first reads nothing overlaps.  (All channels in one workgroup: 5.1 to 5.7 and 34.)
#include "paged.h"

namespace actqkv {

constexpr int kPaThreads = 256;
constexpr int kPaSlices = 2;                                        // of the channels

template <typename T, int D>
__global__ __launch_bounds__(kPaThreads) void paged_append_kernel(PagedTable t, const T* __restrict__ k_new,
                                                                  const T* __restrict__ v_new, T* __restrict__ k_pages,
                                                                  T* __restrict__ v_pages, int n_kv_heads) {
  constexpr int V = Vec<T>::N, kOwn = D / kPaSlices, kChunks = kOwn / V, kPad = kBlock + 2;
  typedef typename Vec<T>::raw raw_t;
  __shared__ __attribute__((aligned(16))) T vt[kOwn * kPad];        // [channel][place in the page]
  const int hk = blockIdx.x / kPaSlices, d0 = blockIdx.x % kPaSlices * kOwn, s = blockIdx.z;
  const PagedSeq q = paged_seq(t, s);
  const int pos0 = q.n - q.m, index = max(pos0, 0) / kBlock + int(blockIdx.y);
  const int lo = max(max(pos0, 0), index * kBlock), hi = min(q.n, index * kBlock + kBlock);
  if (hi <= lo) return;                                             // (index < max_pages: hi > index * kBlock)
  const int page = paged_page(t, s, index);
  if (page < 0) return;
  const int n_tok = hi - lo, j0 = lo - index * kBlock;
  const size_t tile = (size_t(page) * n_kv_heads + hk) * (kBlock * D);
  const size_t src0 = (size_t(q.row0 + (lo - pos0)) * n_kv_heads + hk) * D + d0;
  constexpr int kPairs = kBlock / 2, kEach = kPairs * kChunks / kPaThreads;
  raw_t k[kEach][2], v[kEach][2];
#pragma unroll
  for (int n = 0; n < kEach; ++n) {
    const int i = n * kPaThreads + threadIdx.x, j = i / kChunks * 2, c = i % kChunks;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (j + h >= j0 && j + h < j0 + n_tok) {
        const size_t src = src0 + size_t(j + h - j0) * n_kv_heads * D + c * V;
        k[n][h] = Vec<T>::load_raw(k_new + src);
        v[n][h] = Vec<T>::load_raw(v_new + src);
      } else {
        v[n][h] = raw_t{};
      }
    }
  }
#pragma unroll
  for (int n = 0; n < kEach; ++n) {
    const int i = n * kPaThreads + threadIdx.x, j = i / kChunks * 2, c = i % kChunks;
    if (j + 1 < j0 || j >= j0 + n_tok) continue;
    alignas(16) T ve[2][V];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (j + h >= j0 && j + h < j0 + n_tok) *reinterpret_cast<raw_t*>(k_pages + tile + size_t(j + h) * D + d0 + c * V) = k[n][h];
      *reinterpret_cast<raw_t*>(ve[h]) = v[n][h];
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint32_t*>(vt + (c * V + e) * kPad + j) = uint32_t(ve[0][e]) | uint32_t(ve[1][e]) << 16;
      } else {
        vt[(c * V + e) * kPad + j] = ve[0][e];
        vt[(c * V + e) * kPad + j + 1] = ve[1][e];
      }
    }
  }
  __syncthreads();
  const int g0 = j0 / V, groups = (j0 + n_tok - 1) / V - g0 + 1;
  for (int i = threadIdx.x; i < kOwn * groups; i += kPaThreads) {
    const int d = i / groups, j = (g0 + i - d * groups) * V;
    const T* from = vt + d * kPad + j;
    T* to = v_pages + tile + size_t(d0 + d) * kBlock + j;
    if (j >= j0 && j + V <= j0 + n_tok) {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(from);  // (an even number of elements in)
      *reinterpret_cast<u32x4*>(to) = u32x4{w[0], w[1], w[2], w[3]};
    } else {
      for (int e = max(j0 - j, 0); e < min(V, j0 + n_tok - j); ++e) to[e] = from[e];
    }
  }
}

int launch_paged_append(const actqkv_shape& sh, const PagedTable& t, const void* k_new, const void* v_new,
                        void* k_pages, void* v_pages, hipStream_t stream) {
  // a sequence's rows lie in one page more than they would from a page's first slot on
  const int span = std::min(t.max_pages, (t.max_new + kBlock - 2) / kBlock + 1);
  const dim3 grid(sh.n_kv_heads * kPaSlices, span, t.batch);
  auto launch = [&](auto kernel, auto* type) {
    typedef std::remove_pointer_t<decltype(type)> T;
    hipLaunchKernelGGL(kernel, grid, dim3(kPaThreads), 0, stream, t, static_cast<const T*>(k_new),
                       static_cast<const T*>(v_new), static_cast<T*>(k_pages), static_cast<T*>(v_pages), sh.n_kv_heads);
  };
  if (sh.dtype == ACTQKV_F32) {
    if (sh.head_dim == 64) launch(paged_append_kernel<float, 64>, static_cast<float*>(nullptr));
    else launch(paged_append_kernel<float, 128>, static_cast<float*>(nullptr));
  } else {
    if (sh.head_dim == 64) launch(paged_append_kernel<uint16_t, 64>, static_cast<uint16_t*>(nullptr));
    else launch(paged_append_kernel<uint16_t, 128>, static_cast<uint16_t*>(nullptr));
  }
  return hip_status("paged append");
}

}  // namespace actqkv
