// Which pages a row looks at: the bounds of a page's keys, the score that they give a page for a row, and the selection.
//
// Bounds.  Of every page and KV head the least and the largest key of each channel.  With them sum_d max(q_d lo_d, q_d hi_d) is at least
// every product <q, k> in the page: a page that holds a key that the row answers to is not missed, whatever its other keys are.
// The score of a page for a row and KV head is the largest of that over the G query heads.  Products (exact) and sums are in 64 bits and the result is
// rounded to fp32, so that the order of a sum matters only where 64 bits do not hold it and it lies next to the border of two fp32 numbers: the two ways to
// the scores below, channel by channel and as two sums of positive and of negative queries, differ by a unit of the last place then (by more where a sum cancels).  What is selected
// follows from the scores as they are written.
//
// Scores: a lane has 16 channels of a page, D / 16 lanes a page.  Selection: the key of the last page that stays by a radix histogram, eight bits at a
// time from the highest in which keys differ, then the chosen pages in their order; integers throughout, ties to the lower page.
//
// Bound by the 64-bit sums (26 cycles of a SIMD for 64 products, by the matrix instruction 13 where rows are many) and, of few rows, by the way from the
// last score to the selection: 16 sequences at up to 32K tokens, 32 query and 8 KV heads of 128, 10 us in a graph, 12 alone (in two launches 8.4 + 6.6; 32
// pages a workgroup 16.9, 128 19.6), 4 rows at 128K 14.8 in a graph (15.4 with all four digits and three barriers for each), 512 rows at 100K 151 (332 row
// by row, 305 with the products of bf16 in fp32, which end at 2^128), 142 rows of 6 pages, 28 and 4 heads, 7.4 (12.8 if wavefronts without a page sum all
// the same).  (The key bit by bit in one wavefront's registers: 17, its ballots wait for one another.)  Bounds of the pages with new tokens of 16
// sequences: 3.3 us in a graph, 5 alone, a chain of loads.
#include "paged.h"

namespace actqkv {

constexpr int kSelThreads = 256, kSelWaves = kSelThreads / 64;
constexpr int kSelMostY = 32768;           // workgroups along y: more work goes round
constexpr int kSelEach = 4;                // keys that a thread of the selection holds (of more pages it reads the scores again)
constexpr int kSelWgs = 1024, kSelLeast = 64;   // workgroups that a selection is cut into, of so many pages at least

template <int J>
__device__ __forceinline__ double lane_xor64(double v) {
  const u32x2 x = __builtin_bit_cast(u32x2, v);
  return __builtin_bit_cast(double, u32x2{lane_xor32<J>(x.x), lane_xor32<J>(x.y)});
}

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
  int parts;                               // workgroups of a (row, KV head)
  unsigned int* counters;                  // one of each, zero between launches
};
// A page's place in the order, by its score: 0 is no candidate, the largest one that always stays.
__device__ __forceinline__ uint32_t page_key(const PagedSelect& a, float score, int b, int last) {
  if (score == -INFINITY) return 0;
  if (b < a.keep_first || b > last - a.keep_last) return 0xffffffffu;
  const uint32_t bits = __float_as_uint(score), order = bits >> 31 ? ~bits : bits | 0x80000000u;
  return min(max(order, 1u), 0xfffffffeu);
}
// The selection of one (row, KV head) from the keys of the pages 0 .. last: key_of(i, b) is that of page b = i kSelThreads + threadIdx.x, 0
// behind the last.
template <typename Key>
__device__ __forceinline__ void select_from(const PagedSelect& a, int item, int last, Key key_of) {
  constexpr int kDigits = 4, kAlways = 3;
  __shared__ int hist[kDigits][256], wave_sum[2][kSelEach][kSelWaves];
  __shared__ uint32_t wave_bits[kAlways + 1][kSelWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, rounds = last / kSelThreads + 1;
  int32_t* idx = a.idx + size_t(item) * a.k_sel;
  // ---- candidates, those that always stay, and the bits in which the others differ
  uint32_t any = 0, all = ~0u;
  int n = 0, always = 0;
  for (int i = 0; i < rounds; ++i) {
    const uint32_t k = key_of(i, i * kSelThreads + tid);
    n += __popcll(__ballot(k != 0));
    always += __popcll(__ballot(k == ~0u));
    if (k != 0 && k != ~0u) any |= k, all &= k;
  }
  if (last >= a.k_sel) {                         // (otherwise all stay)
    any |= lane_xor32<1>(any), all &= lane_xor32<1>(all);
    any |= lane_xor32<2>(any), all &= lane_xor32<2>(all);
    any |= lane_xor32<4>(any), all &= lane_xor32<4>(all);
    any |= lane_xor32<8>(any), all &= lane_xor32<8>(all);
    any |= lane_xor32<16>(any), all &= lane_xor32<16>(all);
    any |= lane_xor32<32>(any), all &= lane_xor32<32>(all);
#pragma unroll
    for (int i = 0; i < kDigits; ++i) hist[i][tid] = 0;
  }
  if (lane == 0) {
    wave_bits[0][wave] = any;
    wave_bits[1][wave] = all;
    wave_bits[2][wave] = n;
    wave_bits[kAlways][wave] = always;
  }
  __syncthreads();
  n = always = 0;
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) {
    any |= wave_bits[0][w];
    all &= wave_bits[1][w];
    n += int(wave_bits[2][w]);
    always += int(wave_bits[kAlways][w]);
  }
  const int take = min(n, a.k_sel);
  // ---- the key above which all are taken, and how many of its equals are: from the highest bit in which keys differ, eight at a time
  uint32_t key = 0;                              // (every candidate's key is above 0)
  int left = 0;
  if (n > take) {
    const uint32_t differ = any & ~all;          // (others than those that always stay: more of them than are left to take)
    left = take - always;
    int top = left > 0 ? 32 - __clz(differ) : 0;               // bits that are not known yet
    uint32_t known = top < 32 ? ~0u << top : 0u;
    key = left > 0 ? all & known : 0xfffffffeu;
    for (int digit = 0; top > 0; ++digit) {
      const int shift = max(top - 8, 0);
      for (int i = 0; i < rounds; ++i) {
        const uint32_t k = key_of(i, i * kSelThreads + tid);
        if (k != 0 && k != ~0u && (k & known) == key) atomicAdd(&hist[digit][k >> shift & 255u], 1);
      }
      __syncthreads();
      // from the top: the bin in which the count reaches `left` (each wavefront for itself)
      int mine[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) mine[i] = hist[digit][255 - (4 * lane + i)], sum += mine[i];
      int before = lane_sums(sum) - sum, bin = 0, rest = 0, whole = 0;
      const unsigned long long here = __ballot(before < left && before + sum >= left);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (before < left && before + mine[i] >= left) {
          bin = 255 - (4 * lane + i);
          rest = left - before;
          whole = before + mine[i] == left;
        }
        before += mine[i];
      }
      const int at = __ffsll(here) - 1;
      key |= uint32_t(__builtin_amdgcn_readlane(bin, at)) << shift;
      known |= 255u << shift;
      left = __builtin_amdgcn_readlane(rest, at);
      top = shift;
      if (__builtin_amdgcn_readlane(whole, at) != 0) {      // all of that bin: the other digits do not matter
        key -= key != 0;                         // (a candidate's key is not 0)
        left = 0;
        break;
      }
    }
  }
  // ---- in their order
  int base = 0, equal = 0;                       // taken above the key, and equal to it, before these rounds
  for (int i0 = 0, turn = 0; i0 < rounds; i0 += kSelEach, turn ^= 1) {
    uint32_t k[kSelEach];
    unsigned long long gt[kSelEach], eq[kSelEach];
#pragma unroll
    for (int i = 0; i < kSelEach; ++i) {
      if (i0 + i >= rounds) break;
      k[i] = key_of(i0 + i, (i0 + i) * kSelThreads + tid);
      gt[i] = __ballot(k[i] > key), eq[i] = __ballot(k[i] == key && k[i] != 0);
      if (lane == 0) wave_sum[turn][i][wave] = __popcll(gt[i]) | __popcll(eq[i]) << 16;
    }
    __syncthreads();                             // (two sets of sums: these rounds write the one that the rounds before do not read)
    const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < kSelEach; ++i) {
      if (i0 + i >= rounds) break;
      int g = base, e = equal;
#pragma unroll
      for (int w = 0; w < kSelWaves; ++w) {
        const int sum = wave_sum[turn][i][w];
        if (w < wave) g += sum & 0xffff, e += sum >> 16;
        base += sum & 0xffff, equal += sum >> 16;
      }
      g += __popcll(gt[i] & below), e += __popcll(eq[i] & below);
      if (k[i] > key || (k[i] == key && k[i] != 0 && e < left)) idx[g + min(e, left)] = (i0 + i) * kSelThreads + tid;
    }
  }
  for (int i = take + tid; i < a.k_sel; i += kSelThreads) idx[i] = -1;
  if (tid == 0) a.n_sel[item] = take;
}

// Scores of many rows by the 64-bit matrix instruction, as sum max(q, 0) hi + min(q, 0) lo: a wavefront takes 16 pages for 16 rows of a
// sequence, one query head after the other, and holds of each the largest.  Lane l has page and row l % 16 and the quarter l / 16 of the channels.
// 512 rows at 100K tokens, 32 query and 8 KV heads of 128, 141 us = 46 TFLOP/s (operands widened anew for each head, in 115 registers instead of 190, 147; in
// 128 with some in scratch 206), and the selection 19.
typedef double f64x4 __attribute__((ext_vector_type(4)));
constexpr int kScRows = 16, kScPages = kSelWaves * 16;
template <typename T, int D>
__global__ __launch_bounds__(kSelThreads) void paged_scores_kernel(PagedSelect a) {
  constexpr int V = Vec<T>::N, kOwn = D / 4, kChunks = kOwn / V;
  typedef typename Vec<T>::raw raw_t;
  const int hk = blockIdx.x % a.n_kv_heads, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int s, tile;
  if (!paged_find_tile(a.t, blockIdx.x / a.n_kv_heads, 1, kScRows, s, tile)) return;
  const PagedSeq seq = paged_seq(a.t, s);
  const int own = lane & 15, quarter = lane >> 4;
  const int i_row = min(tile * kScRows + own, seq.m - 1), pos = seq.n - seq.m + i_row, last = pos >= 0 ? pos / kBlock : -1;
  const bool row_there = tile * kScRows + own < seq.m;
  const int most_pos = seq.n - seq.m + min(tile * kScRows + kScRows, seq.m) - 1, tile_last = most_pos >= 0 ? most_pos / kBlock : -1;
  const T* q = static_cast<const T*>(a.q) + (size_t(seq.row0 + i_row) * a.n_kv_heads + hk) * a.group * D + quarter * kOwn;
  float* scores = a.scores + (size_t(seq.row0 + i_row) * a.n_kv_heads + hk) * a.stride;
  for (int b0 = blockIdx.y * kScPages + wave * 16; b0 < a.t.max_pages; b0 += gridDim.y * kScPages) {
    float most[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) most[r] = -INFINITY;
    unsigned long long there = 0;
    if (b0 <= tile_last) {
      const int page = b0 + own <= tile_last ? paged_page(a.t, s, b0 + own) : -1;
      there = __ballot(page >= 0);
      const T* from = static_cast<const T*>(a.bounds) + (size_t(max(page, 0)) * a.n_kv_heads + hk) * (2 * D) + quarter * kOwn;
      raw_t lo[kChunks], hi[kChunks];
#pragma unroll
      for (int c = 0; c < kChunks; ++c) lo[c] = Vec<T>::load_raw(from + c * V), hi[c] = Vec<T>::load_raw(from + D + c * V);
      for (int h = 0; h < a.group; ++h) {
        raw_t x[kChunks];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) x[c] = Vec<T>::load_raw(q + h * D + c * V);
        f64x4 up = {}, down = {};
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          float l[V], u[V], y[V];
          Vec<T>::widen(lo[c], l);
          Vec<T>::widen(hi[c], u);
          Vec<T>::widen(x[c], y);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            up = __builtin_amdgcn_mfma_f64_16x16x4f64(double(u[e]), double(fmaxf(y[e], 0.f)), up, 0, 0, 0);
            down = __builtin_amdgcn_mfma_f64_16x16x4f64(double(l[e]), double(fminf(y[e], 0.f)), down, 0, 0, 0);
          }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) most[r] = fmaxf(most[r], float(up[r] + down[r]));
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {                // (register r of a lane: page 4 r + l / 16, row l % 16)
      const int i = 4 * r + quarter, b = b0 + i;
      if (row_there && b < a.t.max_pages) scores[b] = b <= last && (there >> i & 1) != 0 ? most[r] + 0.f : -INFINITY;
    }
  }
}

// The pages of a (row, KV head) go to `parts` workgroups; the one that is done last selects.  kScored: the scores are there.
template <typename T, int D, bool kScored>
__global__ __launch_bounds__(kSelThreads) void paged_select_kernel(PagedSelect a) {
  constexpr int V = Vec<T>::N, kOwn = 16, kLanes = D / kOwn, kPages = kSelThreads / kLanes;
  __shared__ int last_flag;
  const int item = blockIdx.x / a.parts, part = blockIdx.x - item * a.parts, row = item / a.n_kv_heads, hk = item % a.n_kv_heads;
  const int slice = threadIdx.x % kLanes, at = threadIdx.x / kLanes;
  const int first = __builtin_amdgcn_readfirstlane(at);      // of this wavefront
  const int s = paged_seq_of_row(a.t, row);
  if (s < 0) return;
  const PagedSeq seq = paged_seq(a.t, s);
  const int pos = seq.n - seq.m + (row - seq.row0);
  const int last = pos >= 0 ? pos / kBlock : -1;     // the last page that the row sees (below max_pages: pos < n)
  uint32_t* scores = reinterpret_cast<uint32_t*>(a.scores) + size_t(item) * a.stride;
  if constexpr (!kScored) {
    const T* q = static_cast<const T*>(a.q) + (size_t(row) * a.n_kv_heads + hk) * a.group * D + slice * kOwn;
    constexpr int kAtOnce = 2;
    for (int b0 = part * (kAtOnce * kPages); b0 <= last; b0 += a.parts * (kAtOnce * kPages)) {
      int page[kAtOnce];
      float lo[kAtOnce][kOwn], hi[kAtOnce][kOwn], most[kAtOnce];
#pragma unroll
      for (int n = 0; n < kAtOnce; ++n) page[n] = b0 + n * kPages + at <= last ? paged_page(a.t, s, b0 + n * kPages + at) : -1;
#pragma unroll
      for (int n = 0; n < kAtOnce; ++n) {
        const T* from = static_cast<const T*>(a.bounds) + (size_t(max(page[n], 0)) * a.n_kv_heads + hk) * (2 * D) + slice * kOwn;
        most[n] = -INFINITY;
#pragma unroll
        for (int i = 0; i < kOwn; i += V) {
          Vec<T>::load(from + i, *reinterpret_cast<float(*)[V]>(lo[n] + i));
          Vec<T>::load(from + D + i, *reinterpret_cast<float(*)[V]>(hi[n] + i));
        }
      }
      for (int h = 0; h < a.group; ++h) {
        float x[kOwn];
#pragma unroll
        for (int i = 0; i < kOwn; i += V) Vec<T>::load(q + h * D + i, *reinterpret_cast<float(*)[V]>(x + i));
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) {
          if (b0 + n * kPages + first > last) break;
          double sum[2] = {};
#pragma unroll
          for (int i = 0; i < kOwn; ++i) sum[i & 1] = fma(double(x[i]), double(x[i] > 0.f ? hi[n][i] : lo[n][i]), sum[i & 1]);
          double all = sum[0] + sum[1];
          all += lane_xor64<1>(all);
          all += lane_xor64<2>(all);
          if (kLanes == 8) all += lane_xor64<4>(all);
          most[n] = fmaxf(most[n], float(all));
        }
      }
#pragma unroll
      for (int n = 0; n < kAtOnce; ++n) {
        const int b = b0 + n * kPages + at;
        // (adding 0 leaves no -0: equal scores have equal bits)
        if (slice == 0 && b <= last) st_agent(scores + b, __float_as_uint(page[n] >= 0 ? most[n] + 0.f : -INFINITY));
      }
    }
    for (int b = last + 1 + part * kSelThreads + threadIdx.x; b < a.t.max_pages; b += a.parts * kSelThreads)
      scores[b] = __float_as_uint(-INFINITY);
    if (a.parts > 1) {
      if (!last_of_group(a.counters + item, unsigned(a.parts), &last_flag)) return;
    } else {
      __builtin_amdgcn_s_waitcnt(0);         // (this wavefront's scores have been acknowledged)
      __syncthreads();
    }
  }
  auto from_memory = [&](int, int b) { return b <= last ? page_key(a, __uint_as_float(ld_agent(scores + b)), b, last) : 0u; };
  if (last < kSelThreads * kSelEach) {
    uint32_t k[kSelEach];
#pragma unroll
    for (int i = 0; i < kSelEach; ++i) k[i] = from_memory(i, i * kSelThreads + threadIdx.x);
    select_from(a, item, last, [&](int i, int) {
      uint32_t of = k[0];
#pragma unroll
      for (int j = 1; j < kSelEach; ++j) of = i == j ? k[j] : of;
      return of;
    });
  } else {
    select_from(a, item, last, from_memory);
  }
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
// Which way a call's scores take, and the tiles of 16 rows of the matrix instruction's.
// Both ways' time by their products, of rows as they are and in tiles of 16 (and a launch more): us of one | the other, 32 query and 8 KV heads
// of 128: 512 rows at 100K tokens 332 | 151, 64 56 | 31, 16 23.5 | 20.1, at 16K 8.9 | 18.4, 2 x 2048 rows at 16K 462 | 234, 16 x 8 at 32K 36 | 29.5, 16 x 4
// 17.5 | 28; fp32, 8 and 2 heads of 64, 512 rows at 8K 14.0 | 15.5, 32 at 60K 11.9 | 15.1.
static bool select_scored(const actqkv_shape& sh, const PagedTable& t, int* tiles) {
  const int seqs = std::min(t.batch, t.n_rows);
  *tiles = int(std::min<int64_t>(int64_t(seqs) * ((t.max_new + kScRows - 1) / kScRows), t.n_rows / kScRows + seqs));
  const double products = double(sh.n_q_heads) * sh.head_dim * t.max_pages;     // of a row
  return products * t.n_rows / 4.6e6 > products * *tiles * kScRows / 11.6e6 + 3.;
}
// Workgroups of a (row, KV head) that scores its own pages.
static int select_parts(const actqkv_shape& sh, const PagedTable& t) {
  const int64_t items = int64_t(t.n_rows) * sh.n_kv_heads;
  if (items > int64_t(kTicketCounters)) return 1;
  return int(std::max<int64_t>(1, std::min<int64_t>((t.max_pages + kSelLeast - 1) / kSelLeast, kSelWgs / items)));
}
void paged_select_cut(const actqkv_shape& sh, const PagedTable& t, int32_t* cut) {
  int tiles;
  const bool scored = select_scored(sh, t, &tiles);
  cut[0] = scored ? kScRows : 1;
  cut[1] = scored ? 1 : select_parts(sh, t);
  cut[2] = scored ? 2 : 1;
}
int launch_paged_select(const actqkv_shape& sh, const PagedTable& t, const void* q, const void* bounds, int k_sel, int keep_first,
                        int keep_last, float* scores, int64_t stride, int32_t* idx, int32_t* n_sel, const Workspace& ws, hipStream_t stream) {
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
  const int64_t items = int64_t(t.n_rows) * sh.n_kv_heads;
  a.parts = select_parts(sh, t);
  a.counters = ws.counters();
  int tiles;
  const bool scored = select_scored(sh, t, &tiles);
  auto launch = [&](auto* type, auto dim) {
    typedef std::remove_pointer_t<decltype(type)> T;
    constexpr int D = decltype(dim)::value;
    if (!scored) {
      hipLaunchKernelGGL((paged_select_kernel<T, D, false>), dim3(unsigned(items) * a.parts), dim3(kSelThreads), 0, stream, a);
      return;
    }
    a.parts = 1;
    const dim3 grid(unsigned(tiles) * sh.n_kv_heads, std::min((t.max_pages + kScPages - 1) / kScPages, kSelMostY));
    hipLaunchKernelGGL((paged_scores_kernel<T, D>), grid, dim3(kSelThreads), 0, stream, a);
    hipLaunchKernelGGL((paged_select_kernel<T, D, true>), dim3(unsigned(items)), dim3(kSelThreads), 0, stream, a);
  };
  const std::integral_constant<int, 64> d64;
  const std::integral_constant<int, 128> d128;
  if (sh.dtype == ACTQKV_F32) {
    if (sh.head_dim == 64) launch(static_cast<float*>(nullptr), d64);
    else launch(static_cast<float*>(nullptr), d128);
  } else {
    if (sh.head_dim == 64) launch(static_cast<uint16_t*>(nullptr), d64);
    else launch(static_cast<uint16_t*>(nullptr), d128);
  }
  return hip_status("paged page selection");
}

}  // namespace actqkv
