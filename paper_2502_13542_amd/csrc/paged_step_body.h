// The kernel of the paged attention of few rows: of dense steps (paged_step.hip, where its design and figures are), of steps over an 8-bit
// cache (paged8_step.hip) and of rows that look at selected pages (paged_selected.hip).
#pragma once

#include "decode_shape.h"
#include "paged.h"

namespace actqkv {

constexpr int kStThreads = 512, kStWaves = kStThreads / 64;
// Items that a workgroup has at least: 64 KB.  A compute unit takes some 26 bytes a nanosecond from memory, 10 us for the 32 KB each of
// eight wavefronts; where others are idle a short sequence is spread over them.  700 tokens of 8 query and 2 KV heads of 64 in fp32,
// 8 items of 32 KB a workgroup 13.0 us, 4 9.6, 2 8.8, 1 8.8; 2400 tokens 13.4, 10.1, 9.4, 10.8; in bf16 (16 KB) 8000 tokens 9.9, 9.5, 11.8, 12.2.
static constexpr int step_least(int keys, int d, int elem) { return 65536 / (keys * d * elem * 2); }

struct PagedStep {
  PagedAttn a;
  int n_wg;                  // workgroups per (sequence, KV head)
  uint32_t* part;            // [pair][n_wg][16][D + 2] fp32 bits
  unsigned int* counters;    // one ticket counter per pair, zero between launches
  float* scores;             // [pair][max_new * G][max_pages * 128], units of log2, or NULL
  int weight_rows;           // of the last so many rows of a sequence the scores are kept
  const int32_t* idx;        // [n_rows][Hk][k_sel], the pages that each row looks at, or NULL: all
  const int32_t* n_sel;      // [n_rows][Hk]
  int k_sel;
};
// Operands of an item whose cache is of the queries' type.
template <typename T, int D>
struct StepShape : DcShape<T, D> {
  typedef T elem;
  static constexpr bool kScaled = false;
  static constexpr int kQRegs = DcShape<T, D>::kQ;
  using DcShape<T, D>::kK;
  using DcShape<T, D>::kV;
  using DcShape<T, D>::kSubs;
  __device__ static __forceinline__ void load_q(const T* q, int kq, u32x4 (&qb)[kQRegs]) {
#pragma unroll
    for (int ks = 0; ks < kQRegs; ++ks)
      qb[ks] = *reinterpret_cast<const u32x4*>(q + DcShape<T, D>::q_lane(kq) + ks * DcShape<T, D>::kQStep);
  }
  __device__ static __forceinline__ void scores(const u32x4 (&ka)[kK], const u32x4 (&qb)[kQRegs], float, f32x4 (&sc)[kSubs]) {
    DcShape<T, D>::scores(ka, qb, sc);
  }
  __device__ static __forceinline__ void values(const u32x4 (&va)[kV], const f32x4 (&sc)[kSubs], float, f32x4 (&acc)[D / 16]) {
    DcShape<T, D>::values(va, sc, acc);
  }
};


// out and lse of a column from the merged sum, maximum and output of one channel group.
template <typename T, int D>
__device__ __forceinline__ void step_store(const PagedAttn& p, int row, int head, int d, float o, float l, float m) {
  store_elem(static_cast<T*>(p.out) + (size_t(row) * p.n_q_heads + head) * D + d, l > 0.f ? o / l : 0.f);
  if (d == 0 && p.lse != nullptr) p.lse[size_t(row) * p.n_q_heads + head] = (m + log2f(l)) * kLn2;
}

template <typename S, typename T, int D, bool kCap, bool kBias, bool kSelected, int W = kStWaves>
__device__ __forceinline__ void step_body(const PagedStep& st) {
  typedef typename S::elem C;
  constexpr int kRow = D + 2;
  __shared__ __attribute__((aligned(16))) float lds[W * 16 * kRow];
  __shared__ int last_flag;
  const PagedAttn& p = st.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, kq = lane >> 4;
  const int group = p.n_q_heads / p.n_kv_heads;
  int wg, hk, s, row_at = 0;
  PagedSeq seq;
  if constexpr (kSelected) {                   // a row of its own, of the sequence that holds it
    const int item = blockIdx.x / st.n_wg;
    wg = blockIdx.x - item * st.n_wg;
    hk = item % p.n_kv_heads;
    s = paged_seq_of_row(p.t, item / p.n_kv_heads);
    if (s < 0) return;
    seq = paged_seq(p.t, s);
    row_at = item / p.n_kv_heads - seq.row0;
  } else {
    wg = blockIdx.x, hk = blockIdx.y, s = blockIdx.z;
    seq = paged_seq(p.t, s);
  }
  const int cols = kSelected ? group : seq.m * group;
  if (cols == 0 || cols > 16) return;          // (more: another launch's)
  // ---- this lane's column: columns past the last repeat it, nobody reads what they give
  const int col = min(n, cols - 1), i_row = kSelected ? row_at : col / group, row = seq.row0 + i_row;
  const int head = hk * group + (kSelected ? col : col - i_row * group);
  const int pos = seq.n - seq.m + i_row;
  const PagedSpan v = paged_span(p.f, row, pos, seq.n);
  const uint32_t v_len = v.length();
  const float slope = kBias ? p.f.slopes[head] * kLog2e : 0.f;
  u32x4 qb[S::kQRegs];
  S::load_q(static_cast<const T*>(p.q) + (size_t(row) * p.n_q_heads + head) * D, kq, qb);
  // ---- the items that any column sees: from the numbers alone where rows bring no spans of their own
  int lo, hi;
  if constexpr (kSelected) {
    lo = hi = 0;
  } else if (p.f.row_first == nullptr && p.f.row_end == nullptr) {
    lo = p.f.window > 0 ? max(max(seq.n - seq.m, 0) - p.f.window + 1, 0) : 0;
    hi = seq.n;
  } else {
    lo = v_len != 0 ? v.lo : 0x7fffffff;
    hi = v_len != 0 ? v.hi : 0;
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) {
      lo = min(lo, __shfl_xor(lo, d, 64));
      hi = max(hi, __shfl_xor(hi, d, 64));
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
  }
  constexpr int kPerPage = kBlock / S::kKeys, kLeast = step_least(S::kKeys, D, sizeof(C));
  const int pair = (kSelected ? row : s) * p.n_kv_heads + hk;
  const int it0 = hi > 0 ? lo / S::kKeys : 0;
  const int n_items = kSelected ? min(max(st.n_sel[pair], 0), st.k_sel) * kPerPage : hi > 0 ? (hi + S::kKeys - 1) / S::kKeys - it0 : 0;
  const int wgs = min(max((n_items + kLeast - 1) / kLeast, 1), st.n_wg);
  if (wg >= wgs) return;
  float* score_at = st.scores == nullptr ? nullptr : st.scores + size_t(pair) * (p.t.max_new * group) * (size_t(p.t.max_pages) * kBlock);
  const int vote0 = max(seq.m - st.weight_rows, 0) * group;    // first column whose scores are kept

  float m_run = -INFINITY, l_run = 0.f;
  f32x4 acc[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int stride = wgs * W;
  int my_page = -1, my_index = 0;
  float my_k = 1.f, my_v = 1.f;                // scales of the lane's page
  for (int k = 0, it = n_items < stride ? wave * wgs + wg : wg * W + wave; it < n_items; it += stride, ++k) {
    if ((k & 63) == 0) {                       // the pages of this and the next 63 items
      const int mine = it + lane * stride;
      if constexpr (kSelected) {
        my_index = mine < n_items ? st.idx[size_t(pair) * st.k_sel + mine / kPerPage] : -1;
        my_page = my_index >= 0 && my_index < p.t.max_pages ? paged_page(p.t, s, my_index) : -1;
      } else {
        my_page = mine < n_items ? paged_page(p.t, s, (it0 + mine) / kPerPage) : -1;
      }
      if constexpr (S::kScaled) {
        const size_t at = size_t(max(my_page, 0)) * p.n_kv_heads + hk;
        my_k = p.k_scales[at];
        my_v = p.v_scales[at];
      }
    }
    const int page = __builtin_amdgcn_readlane(my_page, k & 63);
    if (page < 0) continue;
    const int part = (it0 + it) % kPerPage;
    const int kpos0 = kSelected ? __builtin_amdgcn_readlane(my_index, k & 63) * kBlock + part * S::kKeys : (it0 + it) * S::kKeys;
    if (kSelected && (kpos0 >= v.hi || kpos0 + S::kKeys <= v.lo)) continue;
    u32x4 ka[S::kK], va[S::kV];
    {
      const size_t tile = (size_t(page) * p.n_kv_heads + hk) * (size_t(kBlock) * D);
      const C* kbase = static_cast<const C*>(p.k_pages) + tile + size_t(part) * S::kKeys * D + S::k_lane(n, kq);
      const C* vbase = static_cast<const C*>(p.v_pages) + tile + part * S::kKeys + S::v_lane(n, kq);
#pragma unroll
      for (int l = 0; l < S::kK; ++l) ka[l] = *reinterpret_cast<const u32x4*>(kbase + S::k_off(l));
#pragma unroll
      for (int l = 0; l < S::kV; ++l) va[l] = *reinterpret_cast<const u32x4*>(vbase + S::v_off(l));
    }
    __builtin_amdgcn_sched_barrier(0);         // everything is in flight before the first MFMA
    f32x4 sc[S::kSubs];
#pragma unroll
    for (int j = 0; j < S::kSubs; ++j) sc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    S::scores(ka, qb, S::kScaled ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_k), k & 63)) : 1.f, sc);
    float mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < S::kSubs; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int kp = kpos0 + S::key_of(j, i, kq);
        const float x = paged_score<kCap, kBias>(p.f, sc[j][i], slope, abs(pos - kp));
        sc[j][i] = span_holds(kp - v.lo, v_len) ? x : -INFINITY;
        mx = fmaxf(mx, sc[j][i]);
      }
    }
    if (!S::kScaled && !kSelected && score_at != nullptr) {   // through LDS, so that a store instruction writes 1 KB in rows of an item's keys
      float* mine = lds + wave * 16 * kRow;
#pragma unroll
      for (int j = 0; j < S::kSubs; ++j)
        if (n < cols) *reinterpret_cast<f32x4*>(mine + n * S::kKeys + S::key_of(j, 0, kq)) = sc[j];
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      for (int e = vote0 * S::kKeys + lane * 4; e < cols * S::kKeys; e += 256)
        *reinterpret_cast<f32x4*>(score_at + size_t(e / S::kKeys) * (size_t(p.t.max_pages) * kBlock) + kpos0 + e % S::kKeys) =
            *reinterpret_cast<const f32x4*>(mine + e);
      __builtin_amdgcn_wave_barrier();
    }
    const auto larger = [](float x, float y) { return fmaxf(x, y); };
    mx = lane_pair<32>(lane_pair<16>(mx, larger), larger);
    const float m_new = fmaxf(m_run, mx), m_safe = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m_run - m_safe);
    m_run = m_new;
    float psum = 0.f;
#pragma unroll
    for (int j = 0; j < S::kSubs; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sc[j][i] = __builtin_amdgcn_exp2f(sc[j][i] - m_safe);
        psum += sc[j][i];
      }
    l_run = l_run * alpha + psum;              // (this lane's quarter of the keys)
#pragma unroll
    for (int dg = 0; dg < D / 16; ++dg) acc[dg] *= alpha;
    if (kpos0 + S::kKeys > seq.n) {            // slots behind the last token: their values may be anything
#pragma unroll
      for (int l = 0; l < S::kV; ++l) S::clear_behind(va[l], S::v_key(l, kq), seq.n - kpos0);
    }
    S::values(va, sc, S::kScaled ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_v), k & 63)) : 1.f, acc);
  }
  const auto sum = [](float x, float y) { return x + y; };
  l_run = lane_pair<32>(lane_pair<16>(l_run, sum), sum);

  // ---- the wavefronts of the workgroup
  if (n < cols) {
    float* mine = lds + (wave * 16 + n) * kRow;
#pragma unroll
    for (int dg = 0; dg < D / 16; ++dg) {
      float* to = mine + 16 * dg + 4 * kq;     // (rows are an even number of floats: 8-byte stores)
      *reinterpret_cast<f32x2*>(to) = f32x2{acc[dg][0], acc[dg][1]};
      *reinterpret_cast<f32x2*>(to + 2) = f32x2{acc[dg][2], acc[dg][3]};
    }
    if (kq == 0) {
      mine[D] = m_run;
      mine[D + 1] = l_run;
    }
  }
  __syncthreads();
  uint32_t* group_part = st.part + size_t(pair) * st.n_wg * (16 * kRow);
  for (int e = tid; e < cols * D; e += 64 * W) {
    const int c = e / D, d = e % D;
    float m = -INFINITY, l = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, lds[(w * 16 + c) * kRow + D]);
    const float m_safe = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float* from = lds + (w * 16 + c) * kRow;
      const float x = __builtin_amdgcn_exp2f(from[D] - m_safe);
      l = fmaf(x, from[D + 1], l);
      o = fmaf(x, from[d], o);
    }
    if (wgs == 1) {
      step_store<T, D>(p, seq.row0 + (kSelected ? row_at : c / group), hk * group + c % group, d, o, l, m);
    } else {
      uint32_t* to = group_part + (wg * 16 + c) * kRow;
      st_agent(to + d, __float_as_uint(o));
      if (d == 0) {
        st_agent(to + D, __float_as_uint(m));
        st_agent(to + D + 1, __float_as_uint(l));
      }
    }
  }
  if (wgs == 1) return;
  if (!last_of_group(st.counters + pair, unsigned(wgs), &last_flag)) return;
  // ---- the workgroups, in their order (whoever is last)
  for (int e = tid; e < cols * D; e += 64 * W) {
    const int c = e / D, d = e % D;
    const uint32_t* from = group_part + c * kRow;
    float m = -INFINITY, l = 0.f, o = 0.f;
    constexpr int kBatch = 8;
    for (int w0 = 0; w0 < wgs; w0 += kBatch) {
      uint32_t pm[kBatch], pl[kBatch], po[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const uint32_t* at = from + size_t(min(w0 + i, wgs - 1)) * (16 * kRow);
        pm[i] = ld_agent(at + D);
        pl[i] = ld_agent(at + D + 1);
        po[i] = ld_agent(at + d);
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        if (w0 + i < wgs) {
          const float m_of = __uint_as_float(pm[i]), m_new = fmaxf(m, m_of), m_safe = m_new == -INFINITY ? 0.f : m_new;
          const float a = __builtin_amdgcn_exp2f(m - m_safe), b = __builtin_amdgcn_exp2f(m_of - m_safe);
          l = l * a + __uint_as_float(pl[i]) * b;
          o = o * a + __uint_as_float(po[i]) * b;
          m = m_new;
        }
      }
    }
    step_store<T, D>(p, seq.row0 + (kSelected ? row_at : c / group), hk * group + c % group, d, o, l, m);
  }
}


// ---- host side
// Workgroups per (sequence, KV head), or row and KV head, of `items` items at most: as many as fill the compute units once, and more only
// where a wavefront still has `each` items, which evens out sequences of different length; every one adds a part to merge.  us with
// 256 | 1024 workgroups, 32 query and 8 KV heads: 1 sequence at 32K tokens 28 | 41, 4 at 8K 24 | 30, 8 at up to 16K 83 | 88, 16
// at up to 32K 300 | 264 (those take the 1024).  Of 8-bit pages, as many bytes of twice as many keys, eight items are 154 us there, four 148,
// two 167.
inline int step_workgroups(int64_t pairs, int64_t items, int64_t least, int each = 8) {
  if (pairs > int64_t(kTicketCounters)) return 1;
  const int64_t fill = (kChipCus + pairs - 1) / pairs, even = std::min(items / (each * kStWaves), (kStepWgs + pairs - 1) / pairs);
  return int(std::max<int64_t>(1, std::min({std::max(fill, even), (items + least - 1) / least, int64_t(64)})));
}
// Partial results of at most kStepWgs + pairs workgroups.
inline size_t step_part_most(const actqkv_shape& sh, int64_t pairs) {
  const size_t wgs = std::min<size_t>(pairs, kTicketCounters) + kStepWgs;
  return align_up(wgs * 16 * (sh.head_dim + 2) * sizeof(float), 256);
}

}  // namespace actqkv
