// Rotation of keys and queries by their position, on the way into the paged cache.
//
// The first `dims` of a head's channels are taken in pairs (a, b), channels (i, i + dims / 2) or, interleaved, (2 i, 2 i + 1), and pair i
// of a row becomes (a cos - b sin, b cos + a sin) with row `position` of a table [n_positions][2][dims / 2] of cosines, then sines.
//
// A thread turns two 16-byte chunks of a head, the same two of several heads of a row: cosines and sines are read once for all of them.
#pragma once

#include "paged.h"

namespace actqkv {

// Threads of a workgroup: of calls whose sequences bring few rows one wavefront, which has no barriers to wait at and leaves room for the
// other workgroups (a step of 64 sequences, 32 query and 8 KV heads of 128, turned: 6.3 us in workgroups of 256 threads, 5.0 so; into 8 bits 10.6, 5.9).
constexpr int kTurnThreads = 256, kTurnFew = 64;
// Workgroups of a launch: of more items they go round (64 chunks of 2048 rows, 32 query and 8 KV heads of 128, 50 thousand items: 599 us, with a
// workgroup each 594; into 8 bits 657, 674).
constexpr int kTurnMostWgs = 1 << 15;
constexpr int kTurnApart = 256;            // (sequence, KV head) pairs of few rows that are worth a launch

// The work of a call is dealt out in items of a KV head: a sequence has slices of its rows and pages with new tokens, as many as it needs
// (a workgroup for every one that the longest could have would be 784 thousand for a chunk of 2048 tokens beside 1000 steps of 8 KV heads).
struct TurnItems {
  int rows, per_page;                      // of a slice (0: no slices); items of a page
  int least, most;                         // new tokens of the sequences that this launch is for
  int total;                               // of all sequences, at most, times the KV heads
};
__host__ __device__ inline int turn_pages(int pos0, int n) { return n > pos0 ? (n - 1) / kBlock - pos0 / kBlock + 1 : 0; }
inline TurnItems turn_items(const actqkv_shape& sh, const PagedTable& t, int rows, int per_page, int least, int most) {
  const int64_t seqs = std::min(t.batch, t.n_rows / least), n_rows = std::min<int64_t>(t.n_rows, seqs * most);
  int64_t items = per_page * std::min<int64_t>(seqs * std::min(t.max_pages, (most + kBlock - 2) / kBlock + 1), n_rows / kBlock + 2 * seqs);
  if (rows > 0) items += std::min<int64_t>(seqs * ((most + rows - 1) / rows), n_rows / rows + seqs);
  return TurnItems{rows, per_page, least, most, int(items * sh.n_kv_heads)};
}
// Item `item` of a KV head: a sequence, and a slice of its rows, or (from `slices` on) a part of a page; false behind the last one.
struct TurnItem {
  int s, slice, page, part;                // slice or page -1
};
// (kSeqs: sequences of a lane.  A search of 1000 sequences is 4 rounds of loads, of 64 one.)
template <int kSeqs>
__device__ __forceinline__ bool turn_item_of(const PagedTable& t, const TurnItems& of, int item, TurnItem& it) {
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < t.batch; s0 += 64 * kSeqs) {
    int slices[kSeqs], n[kSeqs], all = 0;
#pragma unroll
    for (int k = 0; k < kSeqs; ++k) {
      const int s = s0 + lane * kSeqs + k;
      const PagedSeq q = paged_seq(t, min(s, t.batch - 1));
      const bool some = s < t.batch && q.m >= of.least && q.m <= of.most;
      slices[k] = some && of.rows > 0 ? (q.m + of.rows - 1) / of.rows : 0;
      n[k] = some ? slices[k] + of.per_page * turn_pages(max(q.n - q.m, 0), q.n) : 0;
      all += n[k];
    }
    const int sum = lane_sums(all);
    const unsigned long long mine = __ballot(item < sum);
    if (mine != 0) {
      const int at = __ffsll(mine) - 1;
      item -= __builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(all, at);
      int k_at = 0, first = __builtin_amdgcn_readlane(slices[0], at);
#pragma unroll
      for (int k = 1; k < kSeqs; ++k) {
        const int before = __builtin_amdgcn_readlane(n[k - 1], at);
        if (k_at == k - 1 && item >= before) {
          item -= before;
          k_at = k;
          first = __builtin_amdgcn_readlane(slices[k], at);
        }
      }
      it.s = s0 + at * kSeqs + k_at;
      it.slice = item < first ? item : -1;
      it.page = item < first ? -1 : (item - first) / of.per_page;
      it.part = (item - first) - it.page * of.per_page;
      return true;
    }
    item -= __builtin_amdgcn_readlane(sum, 63);
  }
  return false;
}
__device__ __forceinline__ bool turn_item(const PagedTable& t, const TurnItems& of, int item, TurnItem& it) {
  return t.batch <= 64 ? turn_item_of<1>(t, of, item, it) : turn_item_of<4>(t, of, item, it);
}

// Chunks a thread's pair is made of: their first channels, and whether they turn (behind `dims` they are just two neighbours).
struct TurnPair {
  int a, b;
  bool turns;
};
template <int V>
__device__ __forceinline__ TurnPair turn_pair(const PagedRotation& r, int p) {
  TurnPair c;
  c.turns = p * (2 * V) < r.dims;
  const bool apart = c.turns && !r.interleaved;
  c.a = apart ? p * V : 2 * p * V;
  c.b = apart ? r.dims / 2 + p * V : c.a + V;
  return c;
}
// Cosines and sines of a thread's V pairs at the row's position (clamped to the table).
template <int V>
struct TurnBy {
  alignas(16) float c[V];
  alignas(16) float s[V];
  __device__ __forceinline__ void load(const PagedRotation& r, int row, int pos, int p) {
    const int at = min(max(r.row_pos != nullptr ? r.row_pos[row] : pos, 0), r.n_positions - 1);
    const float* from = r.table + size_t(at) * r.dims + p * V;
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      *reinterpret_cast<f32x4*>(c + i) = *reinterpret_cast<const f32x4*>(from + i);
      *reinterpret_cast<f32x4*>(s + i) = *reinterpret_cast<const f32x4*>(from + r.dims / 2 + i);
    }
  }
};
// W: the type the products are formed in.
template <typename W, int V>
__device__ __forceinline__ void turn(const TurnBy<V>& by, bool interleaved, float (&a)[V], float (&b)[V]) {
  auto one = [](float& x, float& y, float c, float s) {
    const W x0 = x, y0 = y, c0 = c, s0 = s;
    x = float(x0 * c0 - y0 * s0);
    y = float(y0 * c0 + x0 * s0);
  };
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      one(a[2 * i], a[2 * i + 1], by.c[i], by.s[i]);
      one(b[2 * i], b[2 * i + 1], by.c[V / 2 + i], by.s[V / 2 + i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) one(a[i], b[i], by.c[i], by.s[i]);
  }
}
__device__ __forceinline__ f32x4 narrow(const float (&x)[4], f32x4*) { return f32x4{x[0], x[1], x[2], x[3]}; }
__device__ __forceinline__ u32x4 narrow(const float (&x)[8], u32x4*) {
  return u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
}

// Slice `slice` of a sequence's rows: their query heads of KV head hk, and their keys (kKeys), turned.  Products in fp32, each result
// rounded once to the storage type.
template <typename T, int D, int kThreads> constexpr int kTurnRows = kThreads / (D / (2 * Vec<T>::N));   // rows of a slice
template <typename T, int D, int kThreads, bool kKeys>
__device__ __forceinline__ void turn_rows(const PagedTable& t, const PagedRotation& r, const PagedSeq& seq, int s, int hk, int n_kv_heads,
                                          int group, int slice, const T* k_new, T* k_pages, const T* q, T* q_out) {
  constexpr int V = Vec<T>::N, kPairs = D / (2 * V), kRows = kTurnRows<T, D, kThreads>, kHeads = 4;
  typedef typename Vec<T>::raw raw_t;
  const int i = slice * kRows + threadIdx.x / kPairs, p = threadIdx.x % kPairs;
  const int pos = seq.n - seq.m + i, row = seq.row0 + i;
  if (i >= seq.m || pos < 0) return;             // (a row at a negative position is not in the cache)
  const TurnPair at = turn_pair<V>(r, p);
  TurnBy<V> by;
  if (at.turns) by.load(r, row, pos, p);
  auto move = [&](raw_t x, raw_t y, T* to) {
    if (at.turns) {
      float a[V], b[V];
      Vec<T>::widen(x, a);
      Vec<T>::widen(y, b);
      turn<float, V>(by, r.interleaved, a, b);
      x = narrow(a, static_cast<raw_t*>(nullptr));
      y = narrow(b, static_cast<raw_t*>(nullptr));
    }
    *reinterpret_cast<raw_t*>(to + at.a) = x;
    *reinterpret_cast<raw_t*>(to + at.b) = y;
  };
  raw_t ka, kb;
  int page = -1;
  if (kKeys) {
    const T* from = k_new + (size_t(row) * n_kv_heads + hk) * D;
    ka = Vec<T>::load_raw(from + at.a);
    kb = Vec<T>::load_raw(from + at.b);
    page = paged_page(t, s, pos / kBlock);
  }
  if (q != nullptr) {
    const size_t head0 = (size_t(row) * n_kv_heads + hk) * group * D;
    for (int h0 = 0; h0 < group; h0 += kHeads) {
      raw_t x[kHeads], y[kHeads];
#pragma unroll
      for (int h = 0; h < kHeads; ++h) {
        const T* from = q + head0 + min(h0 + h, group - 1) * D;
        x[h] = Vec<T>::load_raw(from + at.a);
        y[h] = Vec<T>::load_raw(from + at.b);
      }
#pragma unroll
      for (int h = 0; h < kHeads; ++h)
        if (h0 + h < group) move(x[h], y[h], q_out + head0 + (h0 + h) * D);
    }
  }
  if (kKeys && page >= 0) move(ka, kb, k_pages + ((size_t(page) * n_kv_heads + hk) * kBlock + pos % kBlock) * D);
}
// Calls launch(T*, D, threads, few, least, most) with the types of a call and the rows of the sequences that a launch is for: few, where those
// are at most a slice; kMost threads otherwise.  Sequences of few rows beside longer ones take a launch of their own if they may be so many
// that in large workgroups, of which a compute unit holds two, they would take longer: 999 single tokens beside a chunk of 2048, 32 query and 8 KV heads of
// 128, in one launch 241 us and 408 into 8 bits, in two 197 and 229.
template <int kMost, typename Launch>
inline void with_turn_types(const actqkv_shape& sh, const PagedTable& t, Launch launch) {
  auto by_rows = [&](auto* type, auto dim) {
    typedef std::remove_pointer_t<decltype(type)> T;
    constexpr int D = decltype(dim)::value, kFewest = kTurnRows<T, D, kTurnFew>, kFew = kTurnRows<T, D, kTurnThreads>;
    const std::integral_constant<int, kTurnFew> few;
    const std::integral_constant<int, kTurnThreads> all;
    const std::integral_constant<int, kMost> most;
    if (t.max_new <= kFewest) {
      launch(type, dim, few, std::true_type(), 1, t.max_new);
      return;
    }
    const int64_t more = std::max<int64_t>(0, int64_t(t.n_rows) - int64_t(t.batch) * kFewest);
    const bool apart = (t.batch - (more + t.max_new - 1) / t.max_new) * sh.n_kv_heads > kTurnApart;
    if (apart) launch(type, dim, few, std::true_type(), 1, kFewest);
    const int least = apart ? kFewest + 1 : 1;
    if (t.max_new <= kFew) launch(type, dim, all, std::true_type(), least, t.max_new);
    else launch(type, dim, most, std::false_type(), least, t.max_new);
  };
  const std::integral_constant<int, 64> d64;
  const std::integral_constant<int, 128> d128;
  if (sh.dtype == ACTQKV_F32) {
    if (sh.head_dim == 64) by_rows(static_cast<float*>(nullptr), d64);
    else by_rows(static_cast<float*>(nullptr), d128);
  } else {
    if (sh.head_dim == 64) by_rows(static_cast<uint16_t*>(nullptr), d64);
    else by_rows(static_cast<uint16_t*>(nullptr), d128);
  }
}
// What the launches of a call have to do: items and workgroups of the largest, and how many launches there are.
template <int kMost, typename Items>
inline void turn_cut(const actqkv_shape& sh, const PagedTable& t, int32_t* cut, Items items_of) {
  cut[0] = cut[1] = cut[2] = 0;
  with_turn_types<kMost>(sh, t, [&](auto* type, auto dim, auto threads, auto, int least, int most) {
    const int total = items_of(type, dim, threads, least, most).total;
    cut[0] = std::max(cut[0], total);
    cut[1] = std::max(cut[1], std::min(total, kTurnMostWgs));
    cut[2] += total > 0;
  });
}

}  // namespace actqkv
