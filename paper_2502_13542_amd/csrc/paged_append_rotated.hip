// Keys and values of a ragged batch's new tokens into their pages, the keys turned by their position on the way and the queries with
// them (the paged form of Sec. 3.1, Eq. (4), of a model with rotary positions).
//
// One launch, two kinds of workgroups: a slice of a sequence's rows for one KV head, its keys and the queries that read it (turn_rows),
// and half of the channels of the values that fall into one page, which go through LDS two neighbouring tokens a word, so that a
// channel's row of the page is written in 16-byte stores where eight (fp32: four) neighbouring tokens are new.  Bound by HBM: 15.4 thousand tokens
// of 16 sequences, 32 query and 8 KV heads of 128, 387 MB in and out, 76 us = 5.1 TB/s, what a plain copy has; a step by its launch and a
// chain of loads (row_start, the row's place, the table): of 64 sequences 5 us, of one, small fp32 model, 3.4.
#include "paged_rotate.h"

namespace actqkv {

constexpr int kArSlices = 2;               // of the channels of the values

struct PagedAppendRotated {
  PagedTable t;
  PagedRotation r;
  const void *k_new, *v_new, *q;           // q may be NULL
  void *k_pages, *v_pages, *q_out;
  int n_kv_heads, group;
  TurnItems items;
};

// kFew: at most kTurnRows new tokens, all in one round.
template <typename T, int D, int kThreads, bool kFew>
__device__ __forceinline__ void append_values(const PagedAppendRotated& a, const PagedSeq& q, int s, int hk, int index, int d0, T* vt) {
  constexpr int V = Vec<T>::N, kOwn = D / kArSlices, kChunks = kOwn / V, kPad = kBlock + 2;
  typedef typename Vec<T>::raw raw_t;
  const int pos0 = q.n - q.m;
  const int lo = max(max(pos0, 0), index * kBlock), hi = min(q.n, index * kBlock + kBlock);
  if (hi <= lo) return;                                             // (index < max_pages: hi > index * kBlock)
  const int page = paged_page(a.t, s, index);
  if (page < 0) return;
  const int n_tok = hi - lo, j0 = lo - index * kBlock;
  const T* v_new = static_cast<const T*>(a.v_new) + (size_t(q.row0 + (lo - pos0)) * a.n_kv_heads + hk) * D + d0;
  T* tile = static_cast<T*>(a.v_pages) + (size_t(page) * a.n_kv_heads + hk) * (kBlock * D) + size_t(d0) * kBlock;
  constexpr int kEach = kFew ? 1 : kBlock / 2 * kChunks / kThreads;
  static_assert(!kFew || (kTurnRows<T, D, kThreads> / 2 + 1) * kChunks <= kThreads, "pairs of as many tokens, wherever they begin");
  const int pair0 = kFew ? j0 / 2 : 0;                              // the first pair with a new token
  raw_t v[kEach][2];
#pragma unroll
  for (int n = 0; n < kEach; ++n) {
    const int i = n * kThreads + threadIdx.x, j = (pair0 + i / kChunks) * 2, c = i % kChunks;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      v[n][h] = j + h >= j0 && j + h < j0 + n_tok ? Vec<T>::load_raw(v_new + size_t(j + h - j0) * a.n_kv_heads * D + c * V) : raw_t{};
  }
#pragma unroll
  for (int n = 0; n < kEach; ++n) {
    const int i = n * kThreads + threadIdx.x, j = (pair0 + i / kChunks) * 2, c = i % kChunks;
    if (j + 1 < j0 || j >= j0 + n_tok) continue;
    alignas(16) T ve[2][V];
#pragma unroll
    for (int h = 0; h < 2; ++h) *reinterpret_cast<raw_t*>(ve[h]) = v[n][h];
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
  for (int i = threadIdx.x; i < kOwn * groups; i += kThreads) {
    const int d = i / groups, j = (g0 + i - d * groups) * V;
    const T* from = vt + d * kPad + j;
    T* to = tile + size_t(d) * kBlock + j;
    if (j >= j0 && j + V <= j0 + n_tok) {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(from);  // (an even number of elements in)
      *reinterpret_cast<u32x4*>(to) = u32x4{w[0], w[1], w[2], w[3]};
    } else {
      for (int e = max(j0 - j, 0); e < min(V, j0 + n_tok - j); ++e) to[e] = from[e];
    }
  }
}

template <typename T, int D, int kThreads, bool kFew>
__global__ __launch_bounds__(kThreads) void paged_append_rotated_kernel(PagedAppendRotated a) {
  constexpr int kOwn = D / kArSlices;
  __shared__ __attribute__((aligned(16))) T vt[kOwn * (kBlock + 2)];   // [channel][place in the page]
  for (int i = blockIdx.x; i < a.items.total; i += gridDim.x) {
    const int hk = i % a.n_kv_heads;
    TurnItem it;
    if (!turn_item(a.t, a.items, i / a.n_kv_heads, it)) return;
    const PagedSeq seq = paged_seq(a.t, it.s);
    if (it.slice >= 0) {
      turn_rows<T, D, kThreads, true>(a.t, a.r, seq, it.s, hk, a.n_kv_heads, a.group, it.slice, static_cast<const T*>(a.k_new),
                                      static_cast<T*>(a.k_pages), static_cast<const T*>(a.q), static_cast<T*>(a.q_out));
    } else {
      append_values<T, D, kThreads, kFew>(a, seq, it.s, hk, max(seq.n - seq.m, 0) / kBlock + it.page, it.part * kOwn, vt);
      __syncthreads();
    }
  }
}

// The items of a launch.
struct RotatedItems {
  const actqkv_shape& sh;
  const PagedTable& t;
  template <typename T, typename Dim, typename Threads>
  TurnItems operator()(T*, Dim, Threads, int least, int most) const {
    return turn_items(sh, t, kTurnRows<T, Dim::value, Threads::value>, kArSlices, least, most);
  }
};
void paged_append_rotated_cut(const actqkv_shape& sh, const PagedTable& t, int32_t* cut) {
  turn_cut<kTurnThreads>(sh, t, cut, RotatedItems{sh, t});
}
int launch_paged_append_rotated(const actqkv_shape& sh, const PagedTable& t, const PagedRotation& r, const void* q, const void* k_new,
                                const void* v_new, void* k_pages, void* v_pages, void* q_out, hipStream_t stream) {
  PagedAppendRotated a;
  a.t = t;
  a.r = r;
  a.q = q;
  a.k_new = k_new;
  a.v_new = v_new;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.q_out = q_out;
  a.n_kv_heads = sh.n_kv_heads;
  a.group = sh.n_q_heads / sh.n_kv_heads;
  with_turn_types<kTurnThreads>(sh, t, [&](auto* type, auto dim, auto threads, auto few, int least, int most) {
    typedef std::remove_pointer_t<decltype(type)> T;
    constexpr int D = decltype(dim)::value, kThreads = decltype(threads)::value;
    a.items = RotatedItems{sh, t}(type, dim, threads, least, most);
    if (a.items.total == 0) return;
    hipLaunchKernelGGL((paged_append_rotated_kernel<T, D, kThreads, decltype(few)::value>), dim3(std::min(a.items.total, kTurnMostWgs)),
                       dim3(kThreads), 0, stream, a);
  });
  return hip_status("paged append (rotated)");
}

}  // namespace actqkv
