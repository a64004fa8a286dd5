// Which pages a row looks at: the bounds of a page's keys, the score that they give a page for a row, and the selection.
//
// Bounds.  Of every page and KV head the least and the largest key of each channel.  With them sum_d max(q_d lo_d, q_d hi_d) is at least
// every product <q, k> in the page: a page that holds a key that the row answers to is not missed, whatever its other keys are.
// The score of a page for a row and KV head is the largest of that over the G query heads.  Products and sums are in 64 bits and the result is
// rounded to fp32, so that the selection does not depend on the order of a sum.
//
// Scores: a lane has 16 channels of a page, D / 16 lanes a page.  Selection: the key of the last page that stays by four digits of a radix
// histogram, then the chosen pages in their order; integers throughout, ties to the lower page.
#include "paged.h"

namespace actqkv {

constexpr int kSelThreads = 256, kSelWaves = kSelThreads / 64;
constexpr int kSelMostY = 32768;           // workgroups along y: more work goes round

// ---- bounds
struct PagedBounds {
  PagedTable t;                            // row_start NULL: all pages of a sequence, not those with new tokens alone
  const void* k_pages;
  void* bounds;                            // [n_pages][Hk][2][D]
  int n_kv_heads, pages;                   // of a sequence, at most
};
template <typename T, int D>
__global__ __launch_bounds__(kSelThreads) void paged_bounds_kernel(PagedBounds a) {
  constexpr int V = Vec<T>::N, kChunks = D / V, kTokens = kSelThreads / kChunks, kEach = kBlock / kTokens;
  __shared__ float lo_lds[kTokens][D + V], hi_lds[kTokens][D + V];
  const int hk = blockIdx.x, s = blockIdx.z, c = threadIdx.x % kChunks, j = threadIdx.x / kChunks;
  int first = 0, n = paged_tokens(a.t, s);
  if (a.t.row_start != nullptr) {
    const PagedSeq seq = paged_seq(a.t, s);
    if (seq.m == 0) return;
    first = max(seq.n - seq.m, 0) / kBlock;
  }
  for (int y = blockIdx.y; y < a.pages; y += gridDim.y) {
    const int index = first + y, here = min(n - index * kBlock, kBlock);
    if (here <= 0) return;
    const int page = paged_page(a.t, s, index);
    if (page < 0) continue;
    const T* tile = static_cast<const T*>(a.k_pages) + (size_t(page) * a.n_kv_heads + hk) * (kBlock * D);
    float lo[V], hi[V];
#pragma unroll
    for (int e = 0; e < V; ++e) lo[e] = INFINITY, hi[e] = -INFINITY;
    typename Vec<T>::raw x[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i)        // (a token behind the last counts as the last)
      x[i] = Vec<T>::load_raw(tile + size_t(min(i * kTokens + j, here - 1)) * D + c * V);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      float k[V];
      Vec<T>::widen(x[i], k);
#pragma unroll
      for (int e = 0; e < V; ++e) lo[e] = fminf(lo[e], k[e]), hi[e] = fmaxf(hi[e], k[e]);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) lo_lds[j][c * V + e] = lo[e], hi_lds[j][c * V + e] = hi[e];
    __syncthreads();
    if (threadIdx.x < 2 * D) {
      const int d = threadIdx.x % D;
      const bool upper = threadIdx.x >= D;
      float v = upper ? hi_lds[0][d] : lo_lds[0][d];
#pragma unroll
      for (int i = 1; i < kTokens; ++i) v = upper ? fmaxf(v, hi_lds[i][d]) : fminf(v, lo_lds[i][d]);
      store_elem(static_cast<T*>(a.bounds) + (size_t(page) * a.n_kv_heads + hk) * (2 * D) + threadIdx.x, v);
    }
    __syncthreads();
  }
}

// ---- scores and selection
struct PagedSelect {
  PagedTable t;
  const void *q, *bounds;
  int n_kv_heads, group;
  int k_sel, keep_first, keep_last;
  float* scores;                           // [n_rows][Hk][stride]
  int64_t stride;
  int32_t *idx, *n_sel;                    // [n_rows][Hk][k_sel], [n_rows][Hk]
};
// Sequence and position of a row; false of a row that no sequence brings.
__device__ __forceinline__ bool row_place(const PagedTable& t, int row, int& s, int& pos) {
  s = paged_seq_of_row(t, row);
  if (s < 0) return false;
  const PagedSeq seq = paged_seq(t, s);
  pos = seq.n - seq.m + (row - seq.row0);
  return true;
}
template <typename T, int D>
__global__ __launch_bounds__(kSelThreads) void paged_scores_kernel(PagedSelect a) {
  constexpr int V = Vec<T>::N, kOwn = 16, kLanes = D / kOwn, kPages = kSelThreads / kLanes, kHeads = 4;
  const int item = blockIdx.x, row = item / a.n_kv_heads, hk = item % a.n_kv_heads;
  const int part = threadIdx.x % kLanes, at = threadIdx.x / kLanes;
  int s, pos;
  if (!row_place(a.t, row, s, pos)) return;
  const int seen = pos >= 0 ? pos / kBlock + 1 : 0;
  float* scores = a.scores + size_t(item) * a.stride;
  const T* q = static_cast<const T*>(a.q) + (size_t(row) * a.n_kv_heads + hk) * a.group * D + part * kOwn;
  for (int b0 = blockIdx.y * kPages; b0 < a.t.max_pages; b0 += gridDim.y * kPages) {
    const int b = b0 + at;
    const int page = b < min(seen, a.t.max_pages) ? paged_page(a.t, s, b) : -1;
    float most = -INFINITY;
    if (page >= 0) {
      const T* from = static_cast<const T*>(a.bounds) + (size_t(page) * a.n_kv_heads + hk) * (2 * D) + part * kOwn;
      float lo[kOwn], hi[kOwn];
#pragma unroll
      for (int i = 0; i < kOwn; i += V) {
        Vec<T>::load(from + i, *reinterpret_cast<float(*)[V]>(lo + i));
        Vec<T>::load(from + D + i, *reinterpret_cast<float(*)[V]>(hi + i));
      }
      for (int h0 = 0; h0 < a.group; h0 += kHeads) {
        double sum[kHeads] = {};
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
          const T* qh = q + min(h0 + h, a.group - 1) * D;
          float x[kOwn];
#pragma unroll
          for (int i = 0; i < kOwn; i += V) Vec<T>::load(qh + i, *reinterpret_cast<float(*)[V]>(x + i));
#pragma unroll
          for (int i = 0; i < kOwn; ++i) sum[h] += double(x[i]) * double(x[i] > 0.f ? hi[i] : lo[i]);
        }
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
#pragma unroll
          for (int d = 1; d < kLanes; d <<= 1) sum[h] += __shfl_xor(sum[h], d, 64);
          most = fmaxf(most, float(sum[h]));
        }
      }
      most += 0.f;                         // (no -0: equal scores have equal bits)
    }
    if (part == 0 && b < a.t.max_pages) scores[b] = most;
  }
}

// A page's place in the order: 0 is no candidate, the largest one that always stays.
__device__ __forceinline__ uint32_t page_key(const PagedSelect& a, const float* scores, int s, int b, int last) {
  if (b > last || paged_page(a.t, s, b) < 0) return 0;
  if (b < a.keep_first || b > last - a.keep_last) return 0xffffffffu;
  const uint32_t bits = __float_as_uint(scores[b]), order = bits >> 31 ? ~bits : bits | 0x80000000u;
  return min(max(order, 1u), 0xfffffffeu);
}
__global__ __launch_bounds__(kSelThreads) void paged_select_kernel(PagedSelect a) {
  __shared__ int hist[256], wave_sum[kSelWaves], bin_lds, left_lds;
  const int item = blockIdx.x, row = item / a.n_kv_heads, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int s, pos;
  if (!row_place(a.t, row, s, pos)) return;
  const float* scores = a.scores + size_t(item) * a.stride;
  int32_t* idx = a.idx + size_t(item) * a.k_sel;
  const int last = pos >= 0 ? min(pos / kBlock, a.t.max_pages - 1) : -1;      // the last visible page
  // ---- candidates
  int n = 0;
  for (int b = tid; b <= last; b += kSelThreads) n += page_key(a, scores, s, b, last) != 0;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) n += __shfl_xor(n, d, 64);
  if (lane == 0) wave_sum[wave] = n;
  __syncthreads();
  n = 0;
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) n += wave_sum[w];
  const int take = min(n, a.k_sel);
  // ---- the key of the last one that is taken, and how many of its equals are
  uint32_t key = 1, above = 0;             // digits found so far, as a key and as a mask
  int left = take;
  if (n > take) {
    key = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kSelThreads) hist[i] = 0;
      __syncthreads();
      for (int b = tid; b <= last; b += kSelThreads) {
        const uint32_t k = page_key(a, scores, s, b, last);
        if (k != 0 && (k & above) == key) atomicAdd(&hist[k >> shift & 255u], 1);
      }
      __syncthreads();
      if (wave == 0) {                     // from the top: the bin in which the count reaches `left`
        int mine[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) mine[i] = hist[255 - (4 * lane + i)], sum += mine[i];
        int before = wave_scan(sum) - sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < left && before + mine[i] >= left) {
            bin_lds = 255 - (4 * lane + i);
            left_lds = left - before;
          }
          before += mine[i];
        }
      }
      __syncthreads();
      key |= uint32_t(bin_lds) << shift;
      above |= 255u << shift;
      left = left_lds;
    }
  } else {
    left = 0;                              // every candidate's key is at least 1: all are above 0
    key = 0;
  }
  // ---- in their order
  int base = 0, equal = 0;                 // taken above the key, and equal to it, before this round
  for (int b0 = 0; b0 <= last; b0 += kSelThreads) {
    const int b = b0 + tid;
    const uint32_t k = page_key(a, scores, s, b, last);
    const unsigned long long gt = __ballot(k > key), eq = __ballot(k == key && k != 0), below = (1ull << lane) - 1;
    __syncthreads();
    if (lane == 0) wave_sum[wave] = __popcll(gt) | __popcll(eq) << 16;
    __syncthreads();
    int g = base, e = equal;
#pragma unroll
    for (int w = 0; w < kSelWaves; ++w) {
      const int sum = wave_sum[w];
      if (w < wave) g += sum & 0xffff, e += sum >> 16;
      base += sum & 0xffff, equal += sum >> 16;
    }
    g += __popcll(gt & below), e += __popcll(eq & below);
    if (k > key || (k == key && k != 0 && e < left)) idx[g + min(e, left)] = b;
  }
  for (int i = take + tid; i < a.k_sel; i += kSelThreads) idx[i] = -1;
  if (tid == 0) a.n_sel[item] = take;
}

// ---- host side
int launch_paged_bounds(const actqkv_shape& sh, const PagedTable& t, const void* k_pages, void* bounds, hipStream_t stream) {
  PagedBounds a;
  a.t = t;
  a.k_pages = k_pages;
  a.bounds = bounds;
  a.n_kv_heads = sh.n_kv_heads;
  a.pages = t.row_start == nullptr ? t.max_pages : std::min(t.max_pages, (t.max_new + kBlock - 2) / kBlock + 1);
  const dim3 grid(sh.n_kv_heads, std::min(a.pages, kSelMostY), t.batch);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kSelThreads), 0, stream, a); };
  if (sh.dtype == ACTQKV_F32) {
    if (sh.head_dim == 64) launch(paged_bounds_kernel<float, 64>);
    else launch(paged_bounds_kernel<float, 128>);
  } else {
    if (sh.head_dim == 64) launch(paged_bounds_kernel<uint16_t, 64>);
    else launch(paged_bounds_kernel<uint16_t, 128>);
  }
  return hip_status("paged key bounds");
}
int launch_paged_select(const actqkv_shape& sh, const PagedTable& t, const void* q, const void* bounds, int k_sel, int keep_first,
                        int keep_last, float* scores, int64_t stride, int32_t* idx, int32_t* n_sel, hipStream_t stream) {
  PagedSelect a;
  a.t = t;
  a.q = q;
  a.bounds = bounds;
  a.n_kv_heads = sh.n_kv_heads;
  a.group = sh.n_q_heads / sh.n_kv_heads;
  a.k_sel = k_sel;
  a.keep_first = keep_first;
  a.keep_last = keep_last;
  a.scores = scores;
  a.stride = stride;
  a.idx = idx;
  a.n_sel = n_sel;
  const unsigned items = unsigned(t.n_rows) * sh.n_kv_heads;
  const int pages = kSelThreads / (sh.head_dim / 16);
  const dim3 grid(items, std::min((t.max_pages + pages - 1) / pages, kSelMostY));
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kSelThreads), 0, stream, a); };
  if (sh.dtype == ACTQKV_F32) {
    if (sh.head_dim == 64) launch(paged_scores_kernel<float, 64>);
    else launch(paged_scores_kernel<float, 128>);
  } else {
    if (sh.head_dim == 64) launch(paged_scores_kernel<uint16_t, 64>);
    else launch(paged_scores_kernel<uint16_t, 128>);
  }
  hipLaunchKernelGGL(paged_select_kernel, dim3(items), dim3(kSelThreads), 0, stream, a);
  return hip_status("paged page selection");
}

}  // namespace actqkv
