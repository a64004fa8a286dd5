// Keys and values of a ragged batch's new tokens into pages held in 8 bits (e4m3.h), the keys turned by their position on the way if
// a rotation is given, and the queries with them.
//
// A workgroup takes the new tokens of one (sequence, KV head) that fall into one page, its keys or its values: it holds them in
// registers, finds the largest of them and with it the page's scale, 2^e with the least e that leaves all of them within 448 2^e.  A
// page that held tokens before keeps its scale, unless the new ones need a larger one: then its old codes are rounded to that.  Rotated keys are
// formed in 64 bits and rounded to fp32 before they become codes, so that a key next to the border between two codes goes to
// the right one.  Values go through LDS four neighbouring tokens a word.  Bound by HBM and, as a page is one workgroup's, by how few there are: 8.7
// thousand tokens of 12 sequences, 28 query and 4 KV heads of 128, 36 MB in and out, 14.6 us = 2.4 TB/s (600 workgroups, one round; of 512
// threads, whose 137 registers leave room for one, 19); 15.4 thousand of 16, 32 and 8 heads, with their queries turned, 347 MB, 90 us = 3.9 TB/s (a
// page's turned keys are 64 fp32 registers a thread); a step of 64 sequences 6 us, of which the queries' rotation hides behind the rest.
#include "e4m3.h"
#include "paged_rotate.h"

namespace actqkv {

struct PagedAppend8 {
  PagedTable t;
  PagedRotation r;
  const void *k_new, *v_new, *q;           // q may be NULL
  void* q_out;
  uint8_t *k_pages, *v_pages;
  float *k_scales, *v_scales;              // [n_pages][Hk]
  int n_kv_heads, group;
  TurnItems items;                         // (of a page: its keys, its values)
};
// The new tokens of a page: slots [j0, j0 + n), the first of them row `row`.
struct NewTokens {
  int page, j0, n, row, pos;
};

// The scale's exponent: the least that the new values' largest and, where the page held tokens, its old scale allow; `again`: the factor
// of the old codes, 1 where nothing changes.  (The old scale goes into the maximum: all threads have read it before one writes the new one.)
template <int kThreads>
__device__ __forceinline__ int page_exponent(float most, const NewTokens& w, float old_scale, float* scale, float* red, float& again) {
  const int old = e4m3_exponent(old_scale);
  if (w.j0 > 0) most = fmaxf(most, e4m3_most(old));
  most = kThreads == 64 ? wave_max(most) : block_max(most, red);
  const int e = e4m3_exponent_for(most);
  again = w.j0 > 0 ? pow2f(max(old - e, -126)) : 1.f;
  if (threadIdx.x == 0) *scale = pow2f(e);
  return e;
}

// kFew: at most kTurnRows new tokens, all in one round.
template <typename T, int D, int kThreads, bool kFew, bool kTurn>
__device__ __forceinline__ void append8_keys(const PagedAppend8& a, const NewTokens& w, int hk, float* red) {
  constexpr int V = Vec<T>::N, kPairs = D / (2 * V), kRows = kTurnRows<T, D, kThreads>, kEach = kFew ? 1 : kBlock / kRows;
  typedef typename Vec<T>::raw raw_t;
  const int p = threadIdx.x % kPairs, j = threadIdx.x / kPairs;       // of the new tokens, j, j + kRows, ...
  const TurnPair at = turn_pair<V>(a.r, p);
  const T* from = static_cast<const T*>(a.k_new) + (size_t(w.row) * a.n_kv_heads + hk) * D;
  raw_t x[kEach][2];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int tok = i * kRows + j;
    if (tok < w.n) {
      x[i][0] = Vec<T>::load_raw(from + size_t(tok) * a.n_kv_heads * D + at.a);
      x[i][1] = Vec<T>::load_raw(from + size_t(tok) * a.n_kv_heads * D + at.b);
    }
  }
  if (w.page < 0) return;
  float* scale = a.k_scales + size_t(w.page) * a.n_kv_heads + hk;
  const float old_scale = *scale;
  // (turned keys are held in fp32; others are widened twice, which leaves room for twice as many workgroups)
  float k[kTurn ? kEach : 1][2][V], most = 0.f;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int tok = i * kRows + j, at_i = kTurn ? i : 0;
    if (tok < w.n) {
      Vec<T>::widen(x[i][0], k[at_i][0]);
      Vec<T>::widen(x[i][1], k[at_i][1]);
      if (kTurn && at.turns) {
        TurnBy<V> by;
        by.load(a.r, w.row + tok, w.pos + tok, p);
        turn<double, V>(by, a.r.interleaved, k[at_i][0], k[at_i][1]);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) most = largest(largest(most, k[at_i][0][e]), k[at_i][1][e]);
    }
  }
  const size_t tile = (size_t(w.page) * a.n_kv_heads + hk) * (kBlock * D);
  float again;
  const float by = pow2f(-page_exponent<kThreads>(most, w, old_scale, scale, red, again));
  if (again != 1.f) {
    for (int i = threadIdx.x; i < w.j0 * (D / 16); i += kThreads) {
      u32x4* to = reinterpret_cast<u32x4*>(a.k_pages + tile) + i;
      u32x4 c = *to;
#pragma unroll
      for (int e = 0; e < 4; ++e) c[e] = e4m3_again(c[e], again);
      *to = c;
    }
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int tok = i * kRows + j;
    if (tok < w.n) {
      uint8_t* to = a.k_pages + tile + size_t(w.j0 + tok) * D;
      typedef std::conditional_t<V == 8, u32x2, uint32_t> codes_t;      // of a chunk
      typedef std::conditional_t<V == 8, u32x4, u32x2> pair_t;
      uint32_t c[2][V / 4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float (&y)[V] = k[kTurn ? i : 0][h];
        if (!kTurn) Vec<T>::widen(x[i][h], y);
#pragma unroll
        for (int e = 0; e < V; e += 4) c[h][e / 4] = e4m3_pack(y[e] * by, y[e + 1] * by, y[e + 2] * by, y[e + 3] * by);
      }
      if (at.b == at.a + V) {
        *reinterpret_cast<pair_t*>(to + at.a) = __builtin_bit_cast(pair_t, c);
      } else {
        *reinterpret_cast<codes_t*>(to + at.a) = __builtin_bit_cast(codes_t, c[0]);
        *reinterpret_cast<codes_t*>(to + at.b) = __builtin_bit_cast(codes_t, c[1]);
      }
    }
  }
}

constexpr int kV8Pad = kBlock / 4 + 1;           // words of a channel in LDS
template <typename T, int D, int kThreads, bool kFew>
__device__ __forceinline__ void append8_values(const PagedAppend8& a, const NewTokens& w, int hk, float* red, uint32_t* vt) {
  constexpr int V = Vec<T>::N, kChunks = D / V, kWords = kBlock / 4 * kChunks, kEach = kFew || kWords < kThreads ? 1 : kWords / kThreads;
  static_assert(!kFew || (kTurnRows<T, D, kThreads> + 6) / 4 * kChunks <= kThreads, "words of as many tokens, wherever they begin");
  const int quad0 = kFew ? w.j0 / 4 : 0;          // the first word with a new token
  typedef typename Vec<T>::raw raw_t;
  const T* from = static_cast<const T*>(a.v_new) + (size_t(w.row) * a.n_kv_heads + hk) * D;
  raw_t x[kEach][4];
  float most = 0.f;
#pragma unroll
  for (int n = 0; n < kEach; ++n) {
    const int i = n * kThreads + threadIdx.x, j = (quad0 + i / kChunks) * 4 - w.j0, c = i % kChunks;
#pragma unroll
    for (int h = 0; h < 4; ++h)
      x[n][h] = j + h >= 0 && j + h < w.n ? Vec<T>::load_raw(from + size_t(j + h) * a.n_kv_heads * D + c * V) : raw_t{};
  }
  if (w.page < 0) return;
  float* scale = a.v_scales + size_t(w.page) * a.n_kv_heads + hk;
  const float old_scale = *scale;
#pragma unroll
  for (int n = 0; n < kEach; ++n)
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      float v[V];
      Vec<T>::widen(x[n][h], v);
#pragma unroll
      for (int e = 0; e < V; ++e) most = largest(most, v[e]);
    }
  uint8_t* tile = a.v_pages + (size_t(w.page) * a.n_kv_heads + hk) * (kBlock * D);
  float again;
  const float by = pow2f(-page_exponent<kThreads>(most, w, old_scale, scale, red, again));
#pragma unroll
  for (int n = 0; n < kEach; ++n) {
    const int i = n * kThreads + threadIdx.x, quad = quad0 + i / kChunks, j = quad * 4 - w.j0, c = i % kChunks;
    if (j + 3 < 0 || j >= w.n) continue;
    float v[4][V];
#pragma unroll
    for (int h = 0; h < 4; ++h) Vec<T>::widen(x[n][h], v[h]);
#pragma unroll
    for (int e = 0; e < V; ++e) vt[(c * V + e) * kV8Pad + quad] = e4m3_pack(v[0][e] * by, v[1][e] * by, v[2][e] * by, v[3][e] * by);
  }
  __syncthreads();
  const int end = w.j0 + w.n, g0 = again != 1.f ? 0 : w.j0 / 16, groups = (end - 1) / 16 - g0 + 1;
  for (int i = threadIdx.x; i < D * groups; i += kThreads) {
    const int d = i / groups, j = (g0 + i - d * groups) * 16;
    const uint32_t* words = vt + d * kV8Pad + j / 4;
    uint8_t* to = tile + size_t(d) * kBlock + j;
    if (j >= w.j0 && j + 16 <= end) {
      *reinterpret_cast<u32x4*>(to) = u32x4{words[0], words[1], words[2], words[3]};
    } else if (again != 1.f) {
      u32x4 c = *reinterpret_cast<const u32x4*>(to);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int slot = j + 4 * e;
        uint32_t old = 0, fresh = 0;             // masks of the word's bytes
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          old |= slot + b < w.j0 ? 0xffu << (8 * b) : 0u;
          fresh |= slot + b >= w.j0 && slot + b < end ? 0xffu << (8 * b) : 0u;
        }
        c[e] = (c[e] & ~(old | fresh)) | (e4m3_again(c[e], again) & old) | (fresh != 0 ? words[e] & fresh : 0u);
      }
      *reinterpret_cast<u32x4*>(to) = c;
    } else {
      for (int b = max(w.j0 - j, 0); b < min(16, end - j); ++b) to[b] = uint8_t(words[b / 4] >> (8 * (b % 4)));
    }
  }
}

template <typename T, int D, int kThreads, bool kFew, bool kTurn>
__global__ __launch_bounds__(kThreads) void paged8_append_kernel(PagedAppend8 a) {
  __shared__ uint32_t vt[D * kV8Pad];            // [channel][four slots]
  __shared__ float red[32];
  for (int i = blockIdx.x; i < a.items.total; i += gridDim.x) {
    const int hk = i % a.n_kv_heads;
    TurnItem it;
    if (!turn_item(a.t, a.items, i / a.n_kv_heads, it)) return;
    const PagedSeq seq = paged_seq(a.t, it.s);
    if (it.slice >= 0) {
      turn_rows<T, D, kThreads, false>(a.t, a.r, seq, it.s, hk, a.n_kv_heads, a.group, it.slice, nullptr, nullptr, static_cast<const T*>(a.q),
                                       static_cast<T*>(a.q_out));
      continue;
    }
    const int pos0 = seq.n - seq.m, index = max(pos0, 0) / kBlock + it.page;
    const int lo = max(max(pos0, 0), index * kBlock), hi = min(seq.n, index * kBlock + kBlock);
    const NewTokens w{paged_page(a.t, it.s, index), lo - index * kBlock, hi - lo, seq.row0 + lo - pos0, lo};
    if (it.part == 0) append8_keys<T, D, kThreads, kFew, kTurn>(a, w, hk, red);
    else append8_values<T, D, kThreads, kFew>(a, w, hk, red, vt);
    __syncthreads();
  }
}

// The items of a launch; of keys and values alone there are no slices of rows.
struct QuantisedItems {
  const actqkv_shape& sh;
  const PagedTable& t;
  bool queries;
  template <typename T, typename Dim, typename Threads>
  TurnItems operator()(T*, Dim, Threads, int least, int most) const {
    return turn_items(sh, t, queries ? kTurnRows<T, Dim::value, Threads::value> : 0, 2, least, most);
  }
};
void paged_append_quantised_cut(const actqkv_shape& sh, const PagedTable& t, bool queries, int32_t* cut) {
  turn_cut<kTurnThreads>(sh, t, cut, QuantisedItems{sh, t, queries});
}
int launch_paged_append_quantised(const actqkv_shape& sh, const PagedTable& t, const PagedRotation& r, const void* q, const void* k_new,
                             const void* v_new, uint8_t* k_pages, uint8_t* v_pages, float* k_scales, float* v_scales, void* q_out,
                             hipStream_t stream) {
  PagedAppend8 a;
  a.t = t;
  a.r = r;
  a.q = q;
  a.k_new = k_new;
  a.v_new = v_new;
  a.q_out = q_out;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.k_scales = k_scales;
  a.v_scales = v_scales;
  a.n_kv_heads = sh.n_kv_heads;
  a.group = sh.n_q_heads / sh.n_kv_heads;
  with_turn_types<kTurnThreads>(sh, t, [&](auto* type, auto dim, auto threads, auto few, int least, int most) {
    typedef std::remove_pointer_t<decltype(type)> T;
    constexpr int D = decltype(dim)::value, kThreads = decltype(threads)::value;
    a.items = QuantisedItems{sh, t, q != nullptr}(type, dim, threads, least, most);
    if (a.items.total == 0) return;
    const dim3 grid(std::min(a.items.total, kTurnMostWgs));
    constexpr bool kFew = decltype(few)::value;
    if (r.table != nullptr) hipLaunchKernelGGL((paged8_append_kernel<T, D, kThreads, kFew, true>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((paged8_append_kernel<T, D, kThreads, kFew, false>), grid, dim3(kThreads), 0, stream, a);
  });
  return hip_status("paged append (8 bits)");
}

}  // namespace actqkv
