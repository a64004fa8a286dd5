// The kernel of the paged attention of chunks and prompts with fp32 queries, over pages in fp32 (paged_chunk_f32.hip, where its design and
// figures are) and in 8 bits (paged8_chunk_f32.hip), and how a call of it is cut.
#pragma once

#include "e4m3.h"
#include "f32_parts.h"
#include "mfma_util.h"
#include "paged.h"
#include "paged_bits.h"
#include "paged_merge.h"

namespace actqkv {

constexpr int kP4Threads = 256, kP4Waves = 4, kP4Rows = 32 * kP4Waves;
constexpr int kP4Part = 8192;                     // one of the three parts of K or V^T of a tile
constexpr int kP4MaxSplits = 32, kP4Slots = 512;  // pieces of a query tile; workgroups that fill the chip
constexpr int kP4SlotsByte = 1024;                // of pages in 8 bits

struct PagedChunkF32 {
  PagedAttn a;
  int tiles, splits;
  void* part;
  PagedBits chosen;
};
template <int D> using ChunkPieceF32 = PagedPiece<kP4Waves, D / 32, 1>;

// kByte: pages in 8 bits.  A code is a bf16 exactly (one part instead of three, and three products instead of six), and the queries' parts
// are truncated, so that none exceeds bf16's range: no value is without parts.
// kChosen: every row sees selected pages alone, as bits (paged_bits.h); tiles of pages that no row of the workgroup selected are left out.
template <int D, bool kCap, bool kBias, bool kByte, bool kChosen>
__device__ __forceinline__ void chunk_f32_body(const PagedChunkF32& c) {
  constexpr int kParts = kByte ? 1 : 3, kVPart0 = kParts;      // parts of a key, and of a value behind them
  constexpr int kKeys = 4096 / D;                   // keys of a tile: 64 or 32
  constexpr int kPerPage = kBlock / kKeys;
  constexpr int kG = kKeys / 32, kDb = D / 32, kQ = D / 16;
  constexpr uint32_t kKRow = D * 2, kVRow = kKeys * 2;   // bytes of a K / V^T row in one of its parts in LDS
  typedef ChunkPieceF32<D> Piece;
  __shared__ __attribute__((aligned(16))) char lds[2 * kParts * kP4Part];   // the parts of K, those of V^T
  // whether a wavefront brought values above kFfMax: [K, V^T][wavefront]
  __shared__ __attribute__((aligned(16))) uint32_t no_parts[2][kP4Waves];
  __shared__ int span_lds[2][kP4Waves];
  __shared__ uint32_t any_bits[kChosen ? kMostBitWords : 1];
  const PagedAttn& p = c.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, half = lane >> 5;
  const int group = p.n_q_heads / p.n_kv_heads;
  const int hk = blockIdx.x % p.n_kv_heads, rest = blockIdx.x / p.n_kv_heads;
  const int split = rest % c.splits, tile = rest / c.splits;
  int s = 0, qtile = 0;
  if (!paged_find_tile(p.t, tile, group, kP4Rows, s, qtile)) return;
  s = __builtin_amdgcn_readfirstlane(s);
  qtile = __builtin_amdgcn_readfirstlane(qtile);
  const PagedSeq seq = paged_seq(p.t, s);

  // ---- this lane's row, and what the wavefront's and the workgroup's rows see
  const int row_end = seq.m * group;
  const int frow0 = qtile * kP4Rows + wave * 32;
  const bool wave_ok = frow0 < row_end, row_ok = frow0 + n < row_end;
  const int frow = min(frow0 + n, row_end - 1);
  const int i_row = frow / group, head = hk * group + (frow - i_row * group);
  const int row = seq.row0 + i_row, pos = seq.n - seq.m + i_row;
  PagedSpan v = paged_span(p.f, row, pos, seq.n);
  const uint32_t v_len = v.length();
  if (v_len == 0) v = PagedSpan{0x7fffffff, 0};
  const float slope = kBias ? p.f.slopes[head] * kLog2e : 0.f;
  const SpanOfRows seen = span_of_rows(v);
  const int lo_any = __builtin_amdgcn_readfirstlane(seen.lo_any);
  const int hi_any = __builtin_amdgcn_readfirstlane(wave_ok ? seen.hi_any : 0);
  const int lo_all = __builtin_amdgcn_readfirstlane(seen.lo_all);
  const int hi_all = __builtin_amdgcn_readfirstlane(seen.hi_all);
  if (lane == 0) {
    span_lds[0][wave] = wave_ok ? lo_any : 0x7fffffff;
    span_lds[1][wave] = hi_any;
  }
  __syncthreads();
  int wg_lo = 0x7fffffff, wg_hi = 0;
#pragma unroll
  for (int w = 0; w < kP4Waves; ++w) {
    wg_lo = min(wg_lo, span_lds[0][w]);
    wg_hi = max(wg_hi, span_lds[1][w]);
  }
  wg_lo = __builtin_amdgcn_readfirstlane(wg_lo);
  wg_hi = __builtin_amdgcn_readfirstlane(wg_hi);
  const int t_first = wg_hi > 0 ? wg_lo / kKeys : 0, n_tiles = wg_hi > 0 ? (wg_hi + kKeys - 1) / kKeys - t_first : 0;
  const int per = max((n_tiles + c.splits - 1) / c.splits, 1);
  if (split > 0 && split * per >= n_tiles) {        // (its place among the pieces says that there is nothing)
    Piece::store_none(Piece::at(c.part, tile * p.n_kv_heads + hk, c.splits, split, wave), -INFINITY, 0.f, lane);
    return;
  }
  int t_begin = t_first + split * per, t_end = min(t_first + n_tiles, t_begin + per);
  auto next_tile = [&](int t) {                     // the first tile from t on that some row sees
    if constexpr (kChosen) {
      if (t >= t_end) return t_end;
      const int page = next_chosen(any_bits, t / kPerPage, (t_end + kPerPage - 1) / kPerPage);
      return min(page == t / kPerPage ? t : page * kPerPage, t_end);
    }
    return t;
  };
  if constexpr (kChosen) {
    const int first = qtile * kP4Rows / group, last = (min((qtile + 1) * kP4Rows, seq.m * group) - 1) / group;
    any_chosen<kP4Threads>(c.chosen, seq.row0 + first, last - first + 1, hk, p.n_kv_heads, any_bits);
    t_begin = next_tile(t_begin);
  }

  // ---- tiles: a wavefront brings a quarter of the rows of K and of V^T into registers, 4 x 1 KB each
  constexpr int kKPer = 1024 / (4 * D), kVPer = 1024 / (4 * kKeys);   // rows of 1 KB in memory
  const int kc = lane % (64 / kKPer), vc = lane % (64 / kVPer);       // 16-byte piece of a row
  const int kr0 = wave * (kKeys / 4) + lane / (64 / kKPer), vr0 = wave * (D / 4) + lane / (64 / kVPer);
  const uint32_t gk = uint32_t(kr0) * (4 * D) + kc * 16, gv = uint32_t(vr0) * (4 * kBlock) + vc * 16;
  // LDS rows are split into 16-byte chunks, XOR-swizzled with a key made of the row so that 16 rows that
  // are read together hit all banks.
  auto k_key = [](int r) { return uint32_t(D == 64 ? (r >> 1) & 7 : r & 15); };
  auto v_key = [](int r) { return uint32_t(D == 64 ? (r >> 1) & 7 : (r >> 2) & 3); };
  // where this lane's pieces go in a part: piece i of K is 2 i (64 channels: 4 i) rows on, of V^T 4 i (8 i), which changes other bits of the
  // key than the lane does
  const uint32_t wk0 = uint32_t(kr0) * kKRow + ((uint32_t(kc >> 1) ^ k_key(kr0)) << 4) + 8 * (kc & 1);
  const uint32_t wv0 = uint32_t(vr0) * kVRow + ((uint32_t(vc >> 1) ^ v_key(vr0)) << 4) + 8 * (vc & 1);
  auto wk = [&](int i) { return (wk0 ^ (uint32_t(2 * i) << 4)) + uint32_t(i * kKPer) * kKRow; };
  auto wv = [&](int i) { return (wv0 ^ (uint32_t(D == 64 ? 2 * i : 2 * i & 3) << 4)) + uint32_t(i * kVPer) * kVRow; };
  const char* kbase = static_cast<const char*>(p.k_pages);
  const char* vbase = static_cast<const char*>(p.v_pages);
  constexpr uint32_t kPageBytes = uint32_t(kBlock) * D * (kByte ? 1 : 4);
  struct Tile { int key0, lo, hi; size_t at; float k_scale, v_scale; };              // first key, the visible span within the tile, its page's offset
  f32x4 xk[4], xv[4];                                        // a tile on its way
  u32x4 ck, cv;                                              // in 8 bits: 16 codes of a key, of a channel
  const int cr = (wave * 1024 + lane * 16) / D, cc = (lane * 16) % D, wr = (wave * 1024 + lane * 16) / kKeys, wc = (lane * 16) % kKeys;
  auto fetch_tile = [&](const Tile& t) {
    const int k0 = t.key0 % kBlock;
    if constexpr (kByte) {
      ck = *reinterpret_cast<const u32x4*>(kbase + t.at + size_t(k0 + cr) * D + cc);
      cv = *reinterpret_cast<const u32x4*>(vbase + t.at + size_t(wr) * kBlock + k0 + wc);
      return;
    }
    const char* kp = kbase + t.at + size_t(k0) * (4 * D) + gk;
    const char* vp = vbase + t.at + size_t(k0) * 4 + gv;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      xk[i] = *reinterpret_cast<const f32x4*>(kp + i * 1024);
      xv[i] = *reinterpret_cast<const f32x4*>(vp + i * kVPer * (4 * kBlock));
    }
  };
  auto too_large = [&](const f32x4 (&x)[4]) {                // whether any of the wavefront's values is (NaN is not)
    float mx = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; j += 2) mx = fmaxf(fmaxf(fabsf(x[i][j]), fabsf(x[i][j + 1])), mx);
    return __any(mx > kFfMax) != 0;
  };
  // the tile in registers -> LDS, in parts; keys that no row of the workgroup sees count as zeros
  auto store_tile = [&](const Tile& t) {
    if constexpr (kByte) {
      if (t.lo > t.key0 || t.hi < t.key0 + kKeys) {
        const bool key = t.key0 + cr >= t.lo && t.key0 + cr < t.hi;
        const int lo = t.lo - t.key0 - wc, hi = t.hi - t.key0 - wc;      // of the 16 values
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t there = 0;
#pragma unroll
          for (int b = 0; b < 4; ++b) there |= 4 * i + b >= lo && 4 * i + b < hi ? 0xffu << (8 * b) : 0u;
          ck[i] = key ? ck[i] : 0u;
          cv[i] &= there;
        }
      }
      char* to_k = lds + uint32_t(cr) * kKRow;
      char* to_v = lds + kVPart0 * kP4Part + uint32_t(wr) * kVRow;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        *reinterpret_cast<u32x4*>(to_k + ((uint32_t(cc / 8 + h) ^ k_key(cr)) << 4)) = e4m3_bf16x8(ck[2 * h], ck[2 * h + 1], t.k_scale);
        *reinterpret_cast<u32x4*>(to_v + ((uint32_t(wc / 8 + h) ^ v_key(wr)) << 4)) = e4m3_bf16x8(cv[2 * h], cv[2 * h + 1], t.v_scale);
      }
      return;
    }
    if (t.lo > t.key0 || t.hi < t.key0 + kKeys) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int kp = t.key0 + kr0 + i * kKPer, vp = t.key0 + 4 * vc;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          xk[i][j] = kp >= t.lo && kp < t.hi ? xk[i][j] : 0.f;
          xv[i][j] = vp + j >= t.lo && vp + j < t.hi ? xv[i][j] : 0.f;
        }
      }
    }
    const bool k_large = too_large(xk), v_large = too_large(xv);
    if (__builtin_expect(v_large, 0)) {                      // the others; these are added by the reader
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) xv[i][j] = fabsf(xv[i][j]) > kFfMax ? 0.f : xv[i][j];
    }
    if (lane == 0) {
      no_parts[0][wave] = k_large;
      no_parts[1][wave] = v_large;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t a[3], b[3];
      ff_split(xk[i][0], xk[i][1], a);
      ff_split(xk[i][2], xk[i][3], b);
#pragma unroll
      for (int j = 0; j < 3; ++j) *reinterpret_cast<u32x2*>(lds + j * kP4Part + wk(i)) = u32x2{a[j], b[j]};
      ff_split(xv[i][0], xv[i][1], a);
      ff_split(xv[i][2], xv[i][3], b);
#pragma unroll
      for (int j = 0; j < 3; ++j) *reinterpret_cast<u32x2*>(lds + (3 + j) * kP4Part + wv(i)) = u32x2{a[j], b[j]};
    }
  };
  // the pages of 64 of the piece's pages at a time, one per lane; a tile without a page has no visible keys
  const int page0 = t_begin / kPerPage, page_end = (t_end + kPerPage - 1) / kPerPage;
  int my_page = -1, have = -1;
  float my_k = 1.f, my_v = 1.f;                              // their scales
  auto tile_at = [&](int t) {
    const int k = t / kPerPage - page0, key0 = t * kKeys;
    if (k >> 6 != have) {
      have = k >> 6;
      const int at = page0 + have * 64 + lane;
      my_page = at < page_end ? paged_page(p.t, s, at) : -1;
      if constexpr (kByte) {
        const size_t of = size_t(max(my_page, 0)) * p.n_kv_heads + hk;
        my_k = p.k_scales[of];
        my_v = p.v_scales[of];
      }
    }
    const int page = __builtin_amdgcn_readlane(my_page, k & 63);
    return Tile{key0, max(wg_lo, key0), page >= 0 ? min(wg_hi, key0 + kKeys) : key0,
                (size_t(max(page, 0)) * p.n_kv_heads + hk) * kPageBytes,
                __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_k), k & 63)),
                __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_v), k & 63))};
  };

  Tile now{0, 0, 0, 0, 1.f, 1.f};
  if (t_begin < t_end) {
    now = tile_at(t_begin);
    fetch_tile(now);
  }
  // ---- the queries: channels 16 j + 8 half .. + 7 of this lane's row times the scale, in parts: scores come in units of log2 then (under
  // a cap, as its tanh's argument)
  const float scale = kCap ? p.f.cap_in : p.f.scale_log2e;
  const float* qrow = static_cast<const float*>(p.q) + (size_t(row) * p.n_q_heads + head) * D;
  u32x4 qp[3][kQ];
  bool q_large;
  {
    f32x4 x[2 * kQ];
    float mx = 0.f;
#pragma unroll
    for (int j = 0; j < kQ; ++j) {
      x[2 * j] = *reinterpret_cast<const f32x4*>(qrow + 16 * j + 8 * half);
      x[2 * j + 1] = *reinterpret_cast<const f32x4*>(qrow + 16 * j + 8 * half + 4);
    }
#pragma unroll
    for (int j = 0; j < 2 * kQ; ++j)
#pragma unroll
      for (int i = 0; i < 4; i += 2) mx = fmaxf(fmaxf(fabsf(x[j][i]), fabsf(x[j][i + 1])), mx);
    q_large = !kByte && __any(mx > kFfMax || mx * scale > kFfMax);
#pragma unroll
    for (int j = 0; j < kQ; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t part[3];
        if constexpr (kByte) ff_cut_scaled(x[2 * j + (i >> 1)][2 * (i & 1)], x[2 * j + (i >> 1)][2 * (i & 1) + 1], scale, part);
        else ff_split_scaled(x[2 * j + (i >> 1)][2 * (i & 1)], x[2 * j + (i >> 1)][2 * (i & 1) + 1], scale, part);
#pragma unroll
        for (int k = 0; k < 3; ++k) qp[k][j][i] = part[k];
      }
  }
  f32x16 acc_o[kDb];
#pragma unroll
  for (int i = 0; i < kDb; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) acc_o[i][j] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;                      // the row's maximum (log2 units), this lane's share of the sum

  const int kn = perm_row(n);                                // the key of this lane's row in the first product
  const uint32_t* row_bits = kChosen ? c.chosen.of(row, hk, p.n_kv_heads) : nullptr;
  uint32_t word = 0;                                         // of 32 pages, which this lane's row sees
  int word_at = -1;
  for (int t = t_begin, t_next; t < t_end; t = t_next) {
    t_next = kChosen ? next_tile(t + 1) : t + 1;
    bool seen_page = true;
    if constexpr (kChosen) {
      const int of = t / kPerPage;
      if (of >> 5 != word_at) word = row_bits[word_at = of >> 5];
      seen_page = (word >> (of & 31) & 1) != 0;
    }
    const uint32_t len = kChosen && !seen_page ? 0u : v_len;
    const int key0 = now.key0, lo = now.lo, hi = now.hi;
    const size_t at_page = now.at;
    if (t > t_begin) __syncthreads();                        // everybody is done with the tile before
    store_tile(now);
    __syncthreads();
    if (t_next < t_end) {
      now = tile_at(t_next);
      fetch_tile(now);
    }
    if (!(hi > lo && lo < hi_any && hi > lo_any) || (kChosen && !__any(seen_page))) continue;  // none of the wavefront's rows sees any of it
    const bool masked = key0 < lo_all || key0 + kKeys > hi_all || (kChosen && !__all(seen_page));
    bool k_large = q_large, v_large = false;
    if constexpr (!kByte) {
      const u32x4 of_k = *reinterpret_cast<const u32x4*>(no_parts[0]), of_v = *reinterpret_cast<const u32x4*>(no_parts[1]);
      k_large |= __any((of_k.x | of_k.y | of_k.z | of_k.w) != 0u);
      v_large = __any((of_v.x | of_v.y | of_v.z | of_v.w) != 0u);
    }
    f32x16 acc_s[kG];
#pragma unroll
    for (int gg = 0; gg < kG; ++gg)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc_s[gg][i] = 0.f;
    bf16x8 kp[2][kParts][kG];                                // a step's operands are requested a step ahead
    auto read_k = [&](int j) {
#pragma unroll
      for (int gg = 0; gg < kG; ++gg) {
        const char* at = lds + uint32_t(gg * 32 + kn) * kKRow + ((uint32_t(2 * j + half) ^ k_key(kn)) << 4);
#pragma unroll
        for (int k = 0; k < kParts; ++k) kp[j & 1][k][gg] = ff_bf16x8(*reinterpret_cast<const u32x4*>(at + k * kP4Part));
      }
    };
    read_k(0);
#pragma unroll
    for (int j = 0; j < kQ; ++j) {
      if (j + 1 < kQ) read_k(j + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < kFfProducts; ++i) {
        if (kFfOf[i][0] >= kParts) continue;
#pragma unroll
        for (int gg = 0; gg < kG; ++gg)
          acc_s[gg] = ff_mfma(kp[j & 1][kFfOf[i][0]][gg], ff_bf16x8(qp[kFfOf[i][1]][j]), acc_s[gg]);
      }
    }
    if (!kByte && __builtin_expect(k_large, 0)) {
      // a key or query without parts: the scores anew in fp32 products, from memory
#pragma unroll
      for (int gg = 0; gg < kG; ++gg)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc_s[gg][i] = 0.f;
      const float* kt = reinterpret_cast<const float*>(kbase + at_page) + size_t(key0 % kBlock + kn) * D + half;
#pragma unroll 1
      for (int ch = 0; ch < D; ch += 2)
#pragma unroll
        for (int gg = 0; gg < kG; ++gg)
          acc_s[gg] = __builtin_amdgcn_mfma_f32_32x32x2f32(kt[gg * 32 * D + ch], qrow[ch + half], acc_s[gg], 0, 0, 0);
#pragma unroll
      for (int gg = 0; gg < kG; ++gg)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc_s[gg][i] *= scale;
    }
    if constexpr (kCap || kBias)                             // (the scale is in the queries)
      paged_scores<kCap, kBias>(p.f, acc_s, 1.f, cap_form(1.f, p.f.cap_log2e), kTanhSmall, slope, float(pos - key0 - 8 * half),
                                [](int g, int i) { return g * 32 + 16 * (i >> 3) + (i & 7); });
    if (masked) {
      const int ahead = key0 + 8 * half - v.lo;
#pragma unroll
      for (int gg = 0; gg < kG; ++gg)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          acc_s[gg][i] = span_holds(ahead + (gg * 32 + 16 * (i >> 3) + (i & 7)), len) ? acc_s[gg][i] : -INFINITY;
    }
    float mx = acc_s[0][0];
#pragma unroll
    for (int gg = 0; gg < kG; ++gg)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, acc_s[gg][i]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    if (!__all(mx <= m_run)) {
      const float m_new = fmaxf(m_run, mx);
      const float alpha = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
      m_run = m_new;
#pragma unroll
      for (int db = 0; db < kDb; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc_o[db][i] *= alpha;
      l_run *= alpha;
    }
    const float m_safe = m_run == -INFINITY ? 0.f : m_run;
    float psum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int gg = 0; gg < kG; ++gg)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        acc_s[gg][i] = __builtin_amdgcn_exp2f(acc_s[gg][i] - m_safe);
        psum[i & 3] += acc_s[gg][i];
      }
    l_run += (psum[0] + psum[1]) + (psum[2] + psum[3]);
#pragma unroll
    for (int st = 0; st < 2 * kG; ++st) {
      u32x4 pp[3];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t part[3];
        ff_split(acc_s[st >> 1][8 * (st & 1) + 2 * i], acc_s[st >> 1][8 * (st & 1) + 2 * i + 1], part);
#pragma unroll
        for (int k = 0; k < 3; ++k) pp[k][i] = part[k];
      }
#pragma unroll
      for (int d0 = 0; d0 < kDb; d0 += 2) {
        bf16x8 vp[kParts][2];
#pragma unroll
        for (int db = 0; db < 2; ++db) {
          const char* at = lds + kVPart0 * kP4Part + uint32_t((d0 + db) * 32 + n) * kVRow + ((uint32_t(2 * st + half) ^ v_key(n)) << 4);
#pragma unroll
          for (int k = 0; k < kParts; ++k) vp[k][db] = ff_bf16x8(*reinterpret_cast<const u32x4*>(at + k * kP4Part));
        }
#pragma unroll
        for (int i = 0; i < kFfProducts; ++i) {
          if (kFfOf[i][0] >= kParts) continue;
#pragma unroll
          for (int db = 0; db < 2; ++db)
            acc_o[d0 + db] = ff_mfma(vp[kFfOf[i][0]][db], ff_bf16x8(pp[kFfOf[i][1]]), acc_o[d0 + db]);
        }
      }
    }
    if (!kByte && __builtin_expect(v_large, 0)) {
      // values without parts went in as zeros; their products in fp32, from memory
      const float* vt = reinterpret_cast<const float*>(vbase + at_page) + size_t(n) * kBlock + key0 % kBlock;
#pragma unroll
      for (int gg = 0; gg < kG; ++gg)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int k = gg * 32 + 16 * (i >> 3) + 8 * half + (i & 7);
          const bool seen = key0 + k >= lo && key0 + k < hi;
#pragma unroll
          for (int db = 0; db < kDb; ++db) {
            const float x = vt[db * 32 * kBlock + k];
            acc_o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(seen && fabsf(x) > kFfMax ? x : 0.f, acc_s[gg][i], acc_o[db], 0, 0, 0);
          }
        }
    }
  }

  const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
  if (c.splits > 1) {
    Piece::store(Piece::at(c.part, tile * p.n_kv_heads + hk, c.splits, split, wave), acc_o, m_run, l_tot, lane);
    return;
  }
  if (!row_ok) return;
  const size_t at = size_t(row) * p.n_q_heads + head;
  const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
  float* op = static_cast<float*>(p.out) + at * D + 4 * half;
#pragma unroll
  for (int db = 0; db < kDb; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<f32x4*>(op + db * 32 + 8 * j) =
          f32x4{acc_o[db][4 * j] * inv, acc_o[db][4 * j + 1] * inv, acc_o[db][4 * j + 2] * inv, acc_o[db][4 * j + 3] * inv};
  if (p.lse != nullptr && half == 0) p.lse[at] = (m_run + log2f(l_tot)) * kLn2;
}
// ---- host side
inline int chunk_f32_tiles(const actqkv_shape& sh, int batch, int n_rows, int max_new) {
  const int64_t group = sh.n_q_heads / sh.n_kv_heads, seqs = std::min(batch, n_rows);
  return int(std::min(seqs * ((int64_t(max_new) * group + kP4Rows - 1) / kP4Rows), int64_t(n_rows) * group / kP4Rows + seqs));
}
// Pieces of a query tile's keys, by these figures, in us: a tile of keys 2.9 (128 channels 3.2), 1.9 times that where two workgroups
// share a compute unit, or one waits for another (of the first rows of a prompt few pieces have keys, and of several sequences some are short); a launch
// to merge 4, and 0.4 a piece.  8 query and 2 KV heads of 64, us with so many pieces: 2 x 2048 rows at 8192 tokens 1 398, 2 361; 2048
// at 2048 2 63, 4 46; 2 x 512 at 4096 4 68, 8 63; 4 x 33 at 2000 16 20, 32 23; 128 at 16384 16 63, 32 46, 64 52.
// In 8 bits a tile is 1.6 and a piece 2 more, pieces may be twice as many, which evens out tiles of different length, and the factors are
// fitted to these: 2 x 2048 rows at 8192 tokens 1 238, 2 205, 4 187, 8 196 (128 channels 490, 457, 458); 20 sequences of up to 100 rows at up to
// 3000 1 87, 3 41, 6 38, 24 48; 2 x 512 at 4096 4 44, 8 42; 2048 at 2048 2 42, 4 34, 8 37; 128 at 16384 8 68, 16 42, 32 34 (54).
inline int chunk_f32_splits(const actqkv_shape& sh, const PagedAttn& p, int tiles, double* took = nullptr) {
  const int64_t items = int64_t(tiles) * sh.n_kv_heads;
  const int keys = 4096 / sh.head_dim;
  const bool byte = p.k_scales != nullptr;
  const double tile_us = byte ? 1.6 : sh.head_dim == 64 ? 2.9 : 3.2;
  int64_t longest = int64_t(p.t.max_pages) * (kBlock / keys);
  if (p.f.window > 0) longest = std::min<int64_t>(longest, (int64_t(p.f.window) + kP4Rows) / keys + 2);
  if (p.f.row_first != nullptr) longest = (longest + 2) / 3;      // (of documents a part, nobody knows which)
  const double own = double(p.t.max_new) / keys, average = double(longest) - std::min<double>(own, double(longest)) / 2.;
  int best = 1;
  double least = 0.;
  for (int splits = 1; splits <= std::min<int64_t>(kP4MaxSplits, longest) && (splits == 1 || items * splits <= (byte ? kP4SlotsByte : kP4Slots)); ++splits) {
    const double busy = double(items) * splits * average / double(longest) / kChipCus * (p.t.batch > 1 ? 0.8 : 1.);
    double us = double((longest + splits - 1) / splits) * tile_us * (1. + 0.9 * std::min(std::max(busy - 1., 0.), 1.));
    if (byte) {                                    // the longest piece, or what a compute unit has in all
      const double pieces = double(items) * splits * (p.t.batch > 1 ? 0.8 : 1.), share = pieces / kChipCus;
      us = std::max((double((longest + splits - 1) / splits) * tile_us + 2.) * (1. + 0.3 * std::min(std::max(share - 1., 0.), 1.)),
                    share * (average / splits * tile_us + 2.) * 0.6 * (p.t.batch > 1 ? 0.7 : 1.));
      if (splits > 1) us += 4. + pieces * (sh.head_dim * kP4Rows * 8) / 3e6;
    } else if (splits > 1) {
      us += 4. + 0.4 * splits;
    }
    if (splits == 1 || us < least) {
      least = us;
      best = splits;
    }
  }
  if (took != nullptr) *took = least;
  return best;
}
// The merge of a call's pieces, where there are several (paged_chunk_f32.hip).
void launch_chunk_f32_merge(int d, const PagedChunkF32& c, hipStream_t stream);

}  // namespace actqkv
