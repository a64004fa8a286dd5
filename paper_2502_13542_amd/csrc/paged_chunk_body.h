// The kernel of the paged attention of chunks and prompts on the matrix cores, over pages in 16 bits (paged_chunk.hip, where its design
// and figures are) and in 8 (paged8_chunk.hip), and how a call of it is cut.
#pragma once

#include "e4m3.h"
#include "mfma_util.h"
#include "paged.h"
#include "paged_bits.h"
#include "paged_merge.h"

namespace actqkv {

constexpr int kPcThreads = 512, kPcWaves = kPcThreads / 64;
constexpr int kPcMaxSplits = 32;
constexpr size_t kPcMostPiecesByte = 1024; // the same of pages in 8 bits: 138 MB
constexpr size_t kPcMostPieces = 512;      // pieces of 256 rows, or as many bytes of smaller ones, that a call leaves to be merged: 69 MB
template <int KS> constexpr int kPcRows = 32 * kPcWaves / KS;
template <int D> constexpr int kPcTileBytes = kBlock * D * 2;            // the keys or the values of a page
template <int D> constexpr int kPcLdsBytes = 2 * 2 * kPcTileBytes<D>;    // 2 stages x (K, V^T)
constexpr float kPcLazyLog2 = 8.f;

struct PagedChunk {
  PagedAttn a;
  int tiles;                 // query tiles that the launch has workgroups for (a bound)
  int splits;                // pieces of a query tile's pages
  void* part;                // pieces [tile][Hk][split]
  PagedBits chosen;
};
template <int D, int KS>
using ChunkPiece = PagedPiece<kPcWaves / KS, (D / 32 > KS ? D / 32 / KS : 1), (D / 32 < KS ? D / 32 : KS)>;

// out (and lse) of a lane's share of a row: o[j][4 i + r] is channel (db0 + j) 32 + 8 i + 4 half + r.
template <int D, int N>
__device__ __forceinline__ void chunk_store(const PagedAttn& p, const f32x16 (&o)[N], int db0, float m, float l, int row,
                                            int head, int half) {
  const size_t at = size_t(row) * p.n_q_heads + head;
  const float inv = l > 0.f ? 1.f / l : 0.f;
  uint16_t* op = static_cast<uint16_t*>(p.out) + at * D + db0 * 32;
#pragma unroll
  for (int db = 0; db < N; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u32x2 v;
      v.x = pack_bf16x2(o[db][4 * j + 0] * inv, o[db][4 * j + 1] * inv);
      v.y = pack_bf16x2(o[db][4 * j + 2] * inv, o[db][4 * j + 3] * inv);
      *reinterpret_cast<u32x2*>(op + db * 32 + 8 * j + 4 * half) = v;
    }
  if (p.lse != nullptr && half == 0 && db0 == 0) p.lse[at] = (m + log2f(l)) * kLn2;
}

// kByte: pages in 8 bits.  Their codes become bf16 between registers and LDS, once for the workgroup, and what follows is what follows
// in 16 bits.  A page is asked for in the second half of the value products two pages ahead of it (the registers of the scores come
// free there), and placed in LDS behind the scores of the page before it.
// kChosen: every row sees selected pages alone, as bits (paged_bits.h).  The workgroup walks the pages that any of its rows selected.
template <int D, int KS, bool kCap, bool kBias, bool kByte, bool kChosen>
__device__ __forceinline__ void chunk_body(const PagedChunk& c) {
  constexpr int kDb = D / 32, kKs = D / 16;      // 32-channel groups of the output, 16-channel steps of a score
  constexpr int kRows = kPcRows<KS>, kRowGroups = kPcWaves / KS;
  constexpr int kNg = 4 / KS;                    // 32-key groups of a page that are this wavefront's
  // a hidden score: finite where it is multiplied by a factor of itself (0 times infinity is no number)
  constexpr float kHidden = kCap && !kBias ? -1e18f : -INFINITY;
  typedef ChunkPiece<D, KS> Piece;
  constexpr uint32_t kTileBytes = kPcTileBytes<D>;
  __shared__ __attribute__((aligned(16))) char lds_b[kPcLdsBytes<D>];
  __shared__ int span_lds[2][kPcWaves];
  __shared__ uint32_t any_bits[kChosen ? kMostBitWords : 1];
  const PagedAttn& p = c.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, half = lane >> 5;
  const int rg = wave % kRowGroups, quarter = wave / kRowGroups;   // its rows, its share of the keys of every page
  const int kb0 = quarter * kNg;
  const int group = p.n_q_heads / p.n_kv_heads;
  const int hk = blockIdx.x % p.n_kv_heads, rest = blockIdx.x / p.n_kv_heads;
  const int tile = rest / c.splits, split = rest - tile * c.splits;
  int s = 0, qtile = 0;
  if (!paged_find_tile(p.t, tile, group, kRows, s, qtile)) return;
  s = __builtin_amdgcn_readfirstlane(s);
  qtile = __builtin_amdgcn_readfirstlane(qtile);
  const PagedSeq seq = paged_seq(p.t, s);

  // ---- fetching a page: each wavefront an eighth of its keys and of its values, 1 KB an instruction
  constexpr int kLoads = D / 32;
  constexpr uint32_t kKRow = D * 2;
  constexpr int kKPerPiece = 1024 / kKRow;
  uint32_t gk[kLoads], gv[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int kr = (kLoads * wave + i) * kKPerPiece + lane / (64 / kKPerPiece);
    const int kc16 = lane % (64 / kKPerPiece);
    gk[i] = uint32_t(kr) * kKRow + (uint32_t(kc16 ^ (D == 128 ? kr & 15 : (kr >> 1) & 7)) << 4);
    const int vr = (kLoads * wave + i) * 4 + (lane >> 4);
    gv[i] = uint32_t(vr) * 256 + (uint32_t((lane & 15) ^ (vr & 15)) << 4);
  }
  const char* kc = static_cast<const char*>(p.k_pages);
  const char* vc = static_cast<const char*>(p.v_pages);
  // 8 bits: each wavefront an eighth of the codes, 1 KB an instruction
  constexpr int kByteLoads = kByte ? D / 64 : 1;
  u32x4 raw_k[kByteLoads], raw_v[kByteLoads];
  uint32_t to_k[kByteLoads], to_v[kByteLoads];             // where they go in LDS as bf16
  if constexpr (kByte) {
#pragma unroll
    for (int i = 0; i < kByteLoads; ++i) {
      const int at = (kByteLoads * wave + i) * 1024 + lane * 16, kr = at / D, vr = at / kBlock;
      to_k[i] = uint32_t(kr) * kKRow + (uint32_t((at % D / 8) ^ (D == 128 ? kr & 15 : (kr >> 1) & 7)) << 4);
      to_v[i] = kTileBytes + uint32_t(vr) * 256 + (uint32_t((at % kBlock / 8) ^ (vr & 15)) << 4);
    }
  }
  auto ask = [&](int page) {
    const size_t off = (size_t(page) * p.n_kv_heads + hk) * (kTileBytes / 2) + wave * (kTileBytes / 16);
    const char* kt = uniform_ptr(kc + off);
    const char* vt = uniform_ptr(vc + off);
#pragma unroll
    for (int i = 0; i < kByteLoads; ++i) {
      raw_k[i] = *reinterpret_cast<const u32x4*>(kt + i * 1024 + lane * 16);
      raw_v[i] = *reinterpret_cast<const u32x4*>(vt + i * 1024 + lane * 16);
    }
  };
  auto place = [&](int stage, float k_scale, float v_scale) {
    char* dst = lds_b + stage * 2 * kTileBytes;
#pragma unroll
    for (int i = 0; i < kByteLoads; ++i) {
      *reinterpret_cast<u32x4*>(dst + to_k[i]) = e4m3_bf16x8(raw_k[i].x, raw_k[i].y, k_scale);
      *reinterpret_cast<u32x4*>(dst + (to_k[i] ^ 16)) = e4m3_bf16x8(raw_k[i].z, raw_k[i].w, k_scale);
      *reinterpret_cast<u32x4*>(dst + to_v[i]) = e4m3_bf16x8(raw_v[i].x, raw_v[i].y, v_scale);
      *reinterpret_cast<u32x4*>(dst + (to_v[i] ^ 16)) = e4m3_bf16x8(raw_v[i].z, raw_v[i].w, v_scale);
    }
  };
  auto fetch = [&](int page, int stage) {
    const size_t off = (size_t(page) * p.n_kv_heads + hk) * kTileBytes;
    const char* kt = uniform_ptr(kc + off);
    const char* vt = uniform_ptr(vc + off);
    char* dst = lds_b + stage * 2 * kTileBytes + wave * (kTileBytes / 8);
    const __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(kt), 0, kTileBytes, 0x00020000);
    const __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(vt), 0, kTileBytes, 0x00020000);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (__attribute__((address_space(3))) void*)(dst + i * 1024), 16, gk[i], 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (__attribute__((address_space(3))) void*)(dst + kTileBytes + i * 1024), 16, gv[i], 0, 0, 0);
    }
  };
  // ---- where rows bring no spans of their own the tile's is known from its numbers, and its first page is asked for before
  // anything of the rows
  int page = -1, t_begin = 0, t_end = 0;
  // the pages of 64 tiles at a time, one per lane
  int my_page = -1;
  float my_k = 1.f, my_v = 1.f;                  // their scales
  int have = -1;                                 // selected pages: which 64 those are
  auto page_of = [&](int t) {
    const int k = t - t_begin;
    if (kChosen ? k >> 6 != have : (k & 63) == 0) {
      have = k >> 6;
      const int at = kChosen ? t_begin + (k & ~63) + lane : t + lane;
      my_page = at < t_end ? paged_page(p.t, s, at) : -1;
      if constexpr (kByte) {
        const size_t at = size_t(max(my_page, 0)) * p.n_kv_heads + hk;
        my_k = p.k_scales[at];
        my_v = p.v_scales[at];
      }
    }
    return __builtin_amdgcn_readlane(my_page, k & 63);
  };
  struct Scales { float k, v; };
  auto scales_of = [&](int t) {                  // of the page that page_of was asked for last
    const int k = (t - t_begin) & 63;
    return Scales{__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_k), k)),
                  __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_v), k))};
  };
  int page_next = -1;                            // 8 bits: the page on its way, and its scales
  Scales now_by{1.f, 1.f}, next_by{1.f, 1.f};
  bool none = false;                             // a piece without pages
  auto piece_of = [&](int lo, int hi) {          // pages of [lo, hi), this piece's [t_begin, t_end)
    const int t_first = hi > 0 ? lo / kBlock : 0, n_tiles = hi > 0 ? (hi + kBlock - 1) / kBlock - t_first : 0;
    const int per = max((n_tiles + c.splits - 1) / c.splits, 1);
    none = split > 0 && split * per >= n_tiles;
    t_begin = t_first + split * per;
    t_end = min(t_first + n_tiles, t_begin + per);
    if (kChosen) t_begin = next_chosen(any_bits, t_begin, t_end);
    if (t_begin < t_end) {
      page = page_of(t_begin);
      if constexpr (kByte) {
        now_by = scales_of(t_begin);
        ask(max(page, 0));
      } else {
        if (page >= 0) fetch(page, 0);
      }
    }
  };
  if constexpr (kChosen) {
    const int first = qtile * kRows / group, last = (min((qtile + 1) * kRows, seq.m * group) - 1) / group;
    any_chosen<kPcThreads>(c.chosen, seq.row0 + first, last - first + 1, hk, p.n_kv_heads, any_bits);
  }
  const bool arrays = p.f.row_first != nullptr || p.f.row_end != nullptr;
  if (!arrays) {
    const int first = qtile * kRows / group, last = (min((qtile + 1) * kRows, seq.m * group) - 1) / group, w0 = seq.n - seq.m;
    piece_of(p.f.window > 0 ? max(max(w0 + first, 0) - p.f.window + 1, 0) : 0, max(w0 + last + 1, 0));
  }

  // ---- this lane's row
  const int row_end = seq.m * group;
  const int frow0 = qtile * kRows + rg * 32;
  const bool wave_ok = frow0 < row_end, row_ok = frow0 + n < row_end;
  const int frow = min(frow0 + n, row_end - 1);
  const int i_row = frow / group, head = hk * group + (frow - i_row * group);
  const int row = seq.row0 + i_row, pos = seq.n - seq.m + i_row;
  PagedSpan v = paged_span(p.f, row, pos, seq.n);
  const uint32_t v_len = v.length();
  if (v_len == 0) v = PagedSpan{0x7fffffff, 0};
  const float slope = kBias ? p.f.slopes[head] * kLog2e : 0.f;
  bf16x8 qreg[kKs];                              // Q^T as B operand: channels 16 ks + 8 half .. + 7
  {
    const uint16_t* qp = static_cast<const uint16_t*>(p.q) + (size_t(row) * p.n_q_heads + head) * D + 8 * half;
#pragma unroll
    for (int ks = 0; ks < kKs; ++ks) qreg[ks] = as_bf16x8(*reinterpret_cast<const u32x4*>(qp + ks * 16));
  }
  // ---- what the wavefront's rows see: any of them [lo_any, hi_any), all of them [lo_all, hi_all)
  const SpanOfRows seen = span_of_rows(v);
  const int lo_any = __builtin_amdgcn_readfirstlane(seen.lo_any);
  const int hi_any = __builtin_amdgcn_readfirstlane(wave_ok ? seen.hi_any : 0);
  const int lo_all = __builtin_amdgcn_readfirstlane(seen.lo_all);
  const int hi_all = __builtin_amdgcn_readfirstlane(seen.hi_all);
  if (arrays) {
    if (lane == 0) {
      span_lds[0][wave] = wave_ok ? lo_any : 0x7fffffff;
      span_lds[1][wave] = hi_any;
    }
    __syncthreads();
    int lo = 0x7fffffff, hi = 0;
#pragma unroll
    for (int w = 0; w < kRowGroups; ++w) {
      lo = min(lo, span_lds[0][w]);
      hi = max(hi, span_lds[1][w]);
    }
    piece_of(__builtin_amdgcn_readfirstlane(lo), __builtin_amdgcn_readfirstlane(hi));
  }
  if (none) {                                    // (its place among the pieces says that there is nothing)
    if (wave < Piece::kWaves)
      Piece::store_none(Piece::at(c.part, tile * p.n_kv_heads + hk, c.splits, split, wave), -INFINITY, 0.f, lane);
    return;
  }

  f32x16 acc_o[kDb];
#pragma unroll
  for (int i = 0; i < kDb; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) acc_o[i][j] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;          // the row's maximum (units of log2), this lane's share of its sum
  if constexpr (kByte) {
    if (t_begin < t_end) place(0, now_by.k, now_by.v);
    if (t_begin + 1 < t_end) {
      page_next = page_of(t_begin + 1);
      next_by = scales_of(t_begin + 1);
      ask(max(page_next, 0));
    }
  } else {
    __builtin_amdgcn_s_waitcnt(0);
  }
  __syncthreads();

  // offsets of this lane's operands in a page: K row perm(n), V^T row n; the swizzle key XOR-ed in
  const int a_row = perm_row(n);
  uint32_t a_off0 = uint32_t(a_row) * kKRow + (uint32_t(half ^ (D == 128 ? a_row & 15 : (a_row >> 1) & 7)) << 4);
  uint32_t v_off0 = uint32_t(n) * 256 + (uint32_t(half ^ (n & 15)) << 4);
  const uint32_t* row_bits = kChosen ? c.chosen.of(row, hk, p.n_kv_heads) : nullptr;
  uint32_t word = 0;                             // of 32 pages, which this lane's row sees
  int word_at = -1, step = 0;
  for (int t = t_begin, t_next; t < t_end; t = t_next, ++step) {
    const int stage = kChosen ? step & 1 : (t - t_begin) & 1;
    t_next = kChosen ? next_chosen(any_bits, t + 1, t_end) : t + 1;
    bool seen_page = true;
    if constexpr (kChosen) {
      if (t >> 5 != word_at) word = row_bits[word_at = t >> 5];
      seen_page = (word >> (t & 31) & 1) != 0;
    }
    const uint32_t len = kChosen && !seen_page ? 0u : v_len;
    asm volatile("" : "+v"(a_off0), "+v"(v_off0));     // (XOR-ed offsets are recomputed, not kept across the loop)
    int page_after = -1;                         // 8 bits: the page behind the next one
    Scales after_by{1.f, 1.f};
    if constexpr (kByte) {
      if (t + 2 < t_end) {
        page_after = page_of(t + 2);
        after_by = scales_of(t + 2);
      }
    } else {
      page_next = t_next < t_end ? page_of(t_next) : -1;
    }
    const int kpos0 = t * kBlock, sub0 = kpos0 + kb0 * 32, sub1 = sub0 + kNg * 32;
    const bool visible = page >= 0 && sub0 < hi_any && sub1 > lo_any && (!kChosen || __any(seen_page) != 0);
    const bool masked = sub0 < lo_all || sub1 > hi_all || (kChosen && !__all(seen_page));
    char* ks_ = lds_b + stage * 2 * kTileBytes;
    char* vs_ = ks_ + kTileBytes;
    if (kpos0 + kBlock > seq.n) {                // slots behind the last token: their values may be anything
      const int end = seq.n - kpos0;
      for (int i = tid; i < D * 16; i += kPcThreads) {
        const int r = i >> 4, key = (i & 15) * 8;
        if (key + 8 > end) {
          u32x4* at = reinterpret_cast<u32x4*>(vs_ + r * 256 + (((i & 15) ^ (r & 15)) << 4));
          u32x4 x = *at;
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] &= (key + 2 * j < end ? 0xffffu : 0u) | (key + 2 * j + 1 < end ? 0xffff0000u : 0u);
          *at = x;
        }
      }
      __syncthreads();
    }
    f32x16 acc_s[kNg];
    if (visible) {
      // ---- S^T = K Q^T, written in issue order: a ring of operands, each read 8 products ahead; the key groups (one alone: two
      // halves of its sum) take turns, so that a product does not wait for the one before it
      const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      constexpr int kChains = kNg == 1 ? 2 : kNg;
      auto k_read = [&](int i) {
        return *reinterpret_cast<const u32x4*>(ks_ + (a_off0 ^ (uint32_t(i / kNg) << 5)) + (kb0 + i % kNg) * 32 * kKRow);
      };
      constexpr int kScore = kNg * kKs, kRing = kScore < 8 ? kScore : 8;
      u32x4 ring[kRing];
      f32x16 acc[kChains];
#pragma unroll
      for (int i = 0; i < kRing; ++i) ring[i] = k_read(i);
#pragma unroll
      for (int i = 0; i < kScore; ++i) {
        const int ch = i % kChains;
        acc[ch] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(ring[i % kRing]), qreg[i / kNg], i < kChains ? zero16 : acc[ch], 0, 0, 0);
        if (i + kRing < kScore) ring[i % kRing] = k_read(i + kRing);
      }
      __builtin_amdgcn_sched_group_barrier(0x100, kRing, 0);
#pragma unroll
      for (int i = 0; i < kScore - kRing; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, kRing, 0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kb = 0; kb < kNg; ++kb) acc_s[kb] = acc[kb];
      if constexpr (kNg == 1) {
#pragma unroll
        for (int i = 0; i < 16; ++i) acc_s[0][i] += acc[1][i];
      }
    }
    // (requested here, not at the top: it has the softmax and the value products of this page to land)
    if constexpr (kByte) {
      if (t + 1 < t_end) place(stage ^ 1, next_by.k, next_by.v);
      if (!visible) ask(max(page_after, 0));
    } else {
      if (page_next >= 0) fetch(page_next, stage ^ 1);
    }
    if (visible) {
      // register i of group kb holds key kpos0 + (kb0 + kb) 32 + 16 (i / 8) + 8 half + i % 8
      CapShort cap;
      if constexpr (kCap && !kBias) {            // the polynomial goes into the exponents below; beyond its range, and where some are hidden, scores are capped here
        cap = cap_short(p.f.cap_in, p.f.cap_log2e);
        const bool small = cap_is_small(acc_s, p.f.cap_in, kTanhShort);
        if (masked || !small) {
#pragma unroll
          for (int kb = 0; kb < kNg; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float x = acc_s[kb][i];
              acc_s[kb][i] = small ? x * cap.factor(x) : paged_tanh(x * p.f.cap_in, p.f.cap_log2e);
            }
          cap = CapShort{1.f, 0.f, 0.f};
        }
      }
      if constexpr (kBias)
        paged_scores<kCap, kBias>(p.f, acc_s, kCap ? p.f.cap_in : p.f.scale_log2e, cap_short(p.f.cap_in, p.f.cap_log2e), kTanhShort, slope,
                                  float(pos - sub0 - 8 * half),
                                  [](int g, int i) { return g * 32 + 16 * (i >> 3) + (i & 7); });
      if (masked) {
        const int ahead = sub0 + 8 * half - v.lo;
#pragma unroll
        for (int kb = 0; kb < kNg; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            acc_s[kb][i] = span_holds(ahead + (kb * 32 + 16 * (i >> 3) + (i & 7)), len) ? acc_s[kb][i] : kHidden;
      }
      // ---- online softmax, one row per lane (lanes n and n + 32 share it)
      auto v_read = [&](int j) {
        return *reinterpret_cast<const u32x4*>(vs_ + (v_off0 ^ (uint32_t(2 * kb0 + j / kDb) << 5)) + (j % kDb) * 32 * 256);
      };
      constexpr int kValue = 2 * kNg * kDb, kVRing = kValue < 8 ? kValue : 8;
      u32x4 vring[kVRing];
#pragma unroll
      for (int i = 0; i < kVRing; ++i) vring[i] = v_read(i);
      float mx = acc_s[0][0];
#pragma unroll
      for (int kb = 0; kb < kNg; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, acc_s[kb][i]);
      mx = lane_pair<32>(mx, [](float x, float y) { return fmaxf(x, y); });
      float m_tile = kBias ? mx : mx * p.f.scale_log2e;
      if constexpr (kCap && !kBias) m_tile = mx == kHidden ? -INFINITY : mx * cap.factor(mx);
      const float m_new = m_tile - m_run > kPcLazyLog2 ? m_tile : m_run;
      const float m_safe = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_safe);
      m_run = m_new;
      if (!__all(alpha == 1.f)) {
#pragma unroll
        for (int db = 0; db < kDb; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc_o[db][i] *= alpha;
        l_run *= alpha;
      }
      auto prob = [&](float x) {
        if constexpr (kBias) return __builtin_amdgcn_exp2f(x - m_safe);
        else if constexpr (kCap) return __builtin_amdgcn_exp2f(fmaf(x, cap.factor(x), -m_safe));
        else return __builtin_amdgcn_exp2f(fmaf(x, p.f.scale_log2e, -m_safe));
      };
#pragma unroll
      for (int i = 0; i < 16; ++i) acc_s[0][i] = prob(acc_s[0][i]);
      __builtin_amdgcn_sched_barrier(0);
      // ---- O^T += V^T P^T in issue order: the exponentials of the next 32 keys between the products of these
      float psum[2] = {0.f, 0.f};
#pragma unroll
      for (int g8 = 0; g8 < 2 * kNg; ++g8) {
        const int kb = g8 >> 1, s2 = g8 & 1;
        if (kByte && g8 == kNg) ask(max(page_after, 0));
        const bf16x8 pb = pack8(acc_s[kb][8 * s2 + 0], acc_s[kb][8 * s2 + 1], acc_s[kb][8 * s2 + 2],
                                acc_s[kb][8 * s2 + 3], acc_s[kb][8 * s2 + 4], acc_s[kb][8 * s2 + 5],
                                acc_s[kb][8 * s2 + 6], acc_s[kb][8 * s2 + 7]);
#pragma unroll
        for (int i = 0; i < 8; ++i) psum[i & 1] += acc_s[kb][8 * s2 + i];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int db = 0; db < kDb; ++db) {
          if (kb < kNg - 1) {
            constexpr int kExp = 8 / kDb;
#pragma unroll
            for (int i = 8 * s2 + kExp * db; i < 8 * s2 + kExp * (db + 1); ++i) acc_s[kb + 1][i] = prob(acc_s[kb + 1][i]);
          }
          __builtin_amdgcn_sched_barrier(0);
          const int j = kDb * g8 + db;
          acc_o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(vring[j % kVRing]), pb, acc_o[db], 0, 0, 0);
          if (j + kVRing < kValue) vring[j % kVRing] = v_read(j + kVRing);
        }
      }
      l_run += psum[0] + psum[1];
    }
    page = page_next;
    if constexpr (kByte) {
      page_next = page_after;
      next_by = after_by;
    } else {
      __builtin_amdgcn_s_waitcnt(0);             // this wavefront's share of the next page has landed in LDS
    }
    __syncthreads();
  }

  // ---- the wavefronts that share rows merge in LDS: each takes over kMine of the 32-channel groups
  float l_tot = lane_pair<32>(l_run, [](float x, float y) { return x + y; });
  constexpr int kMine = kDb > KS ? kDb / KS : 1;
  f32x16 acc_f[kMine];
  const int db0 = quarter * kMine;
  const bool has_mine = db0 < kDb;
  if constexpr (KS == 1) {
#pragma unroll
    for (int db = 0; db < kDb; ++db) acc_f[db] = acc_o[db];
  } else {
    __shared__ float ml_lds[kPcWaves][2][32];
    f32x4* o_lds = reinterpret_cast<f32x4*>(lds_b);   // [wavefront][channel group][register / 4][lane]
#pragma unroll
    for (int db = 0; db < kDb; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        o_lds[((wave * kDb + db) * 4 + i) * 64 + lane] =
            f32x4{acc_o[db][4 * i], acc_o[db][4 * i + 1], acc_o[db][4 * i + 2], acc_o[db][4 * i + 3]};
    if (half == 0) {
      ml_lds[wave][0][n] = m_run;
      ml_lds[wave][1][n] = l_tot;
    }
    __syncthreads();
    float m_of[KS], l_of[KS], m_all = -INFINITY;
#pragma unroll
    for (int w = 0; w < KS; ++w) {
      m_of[w] = ml_lds[w * kRowGroups + rg][0][n];
      l_of[w] = ml_lds[w * kRowGroups + rg][1][n];
      m_all = fmaxf(m_all, m_of[w]);
    }
    const float m_ref = m_all == -INFINITY ? 0.f : m_all;
    l_tot = 0.f;
#pragma unroll
    for (int db = 0; db < kMine; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc_f[db][i] = 0.f;
#pragma unroll
    for (int w = 0; w < KS; ++w) {
      const float weight = __builtin_amdgcn_exp2f(m_of[w] - m_ref);
      l_tot += weight * l_of[w];
      if (has_mine) {
#pragma unroll
        for (int db = 0; db < kMine; ++db)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x4 o = o_lds[(((w * kRowGroups + rg) * kDb + db0 + db) * 4 + i) * 64 + lane];
#pragma unroll
            for (int r = 0; r < 4; ++r) acc_f[db][4 * i + r] += weight * o[r];
          }
      }
    }
    m_run = m_all;
  }
  if (c.splits == 1) {
    if (row_ok && has_mine) chunk_store<D, kMine>(p, acc_f, db0, m_run, l_tot, row, head, half);
    return;
  }
  if (has_mine)
    Piece::store(Piece::at(c.part, tile * p.n_kv_heads + hk, c.splits, split, wave), acc_f, m_run, l_tot, lane);
}
// ---- host side
// The cut of a call: KS, and the pieces of a query tile's pages, by these figures, in us: a page with 256, 128, 64 rows, a tile's start
// and end, and what pieces cost (a launch, and their way out and back at 4 TB/s).  Whole tiles, dealt out as compute units come
// free, from the longest on: the busiest unit has no more than an average one, or the longest tile, if tiles differ, and a whole
// number of rounds if they do not.  (Shares of the pages equal to a page, made by a plan on the device, were slower nearly
// everywhere: 2048 rows at 2048 tokens 52 us | 68.  A tile costs 6 us beside its pages, a cut of one 135 KB out and in.)
// Pieces may be more than run at once: 22 sequences of up to 215 rows at up to 18K tokens, 8 and 2 heads of 128, 213 us, in at most 256
// pieces 270; of 64, 144 | 187.
//   2 x 2048 rows at 16K tokens, 32 query and 8 KV heads of 128: KS 1 908, 2 1036, 4 1563; 1 x 2048 at 2048 59, 52, 75; 8 x 512 at 512
//   49, 59, 86; 512 at 512 21.5, 16.6, 14.4; 12 sequences of up to 500 with a window, 28 and 4 heads 291, 259, 354; 4 of up to 777
//   248, 271, 380; 64 channels, 8192 at 8192 137, 100, 137, with documents 79, 52, 61
// In 8 bits the pages of fewer rows cost more (each is converted by the workgroup), pieces may be twice as many, and the factors are fitted to 14 calls
// at all cuts, of which the chosen one is 2 % from the best on average: 12 sequences of up to 500 rows under a cap and a window KS 1 289, in two 259, KS 2
// 289; without, 380, 341, 379; 22 of up to 215 at up to 18K KS 1 472, in three 204, in eight 180.
struct ChunkCut {
  int ks, splits, tiles;
  double us;                 // by those figures
};
inline int chunk_tiles(const actqkv_shape& sh, int batch, int n_rows, int max_new, int ks) {
  // every sequence's last tile may be partly empty
  const int64_t rows = kPcRows<1> / ks, group = sh.n_q_heads / sh.n_kv_heads, seqs = std::min(batch, n_rows);
  const int64_t most = seqs * ((int64_t(max_new) * group + rows - 1) / rows);
  return int(std::min(most, int64_t(n_rows) * group / rows + seqs));
}
template <int D>
inline size_t chunk_piece_bytes(int ks) {
  return ks == 1 ? ChunkPiece<D, 1>::bytes() : ks == 2 ? ChunkPiece<D, 2>::bytes() : ChunkPiece<D, 4>::bytes();
}
inline size_t chunk_piece_bytes(const actqkv_shape& sh, int ks) {
  return sh.head_dim == 64 ? chunk_piece_bytes<64>(ks) : chunk_piece_bytes<128>(ks);
}
inline ChunkCut chunk_cut(const actqkv_shape& sh, const PagedAttn& p) {
  constexpr double kPageUs[2][2][3] = {{{3.5, 2.0, 1.5}, {2.1, 1.45, 1.0}}, {{3.5, 2.3, 1.75}, {2.1, 1.45, 1.0}}};
  const bool byte = p.k_scales != nullptr;
  const double item_us = byte ? 4. : 5.;
  const PagedTable& t = p.t;
  // pages of the longest tile and of an average one: of a prompt half of its own on average; of documents a part, nobody knows which
  double longest = t.max_pages, own = double(t.max_new) / kBlock;
  if (p.f.window > 0) longest = std::min(longest, p.f.window / double(kBlock) + 2.);
  double average = longest - std::min(own, longest) / 2.;
  bool equal = p.f.window > 0 ? longest < t.max_pages : own * 4. < longest;
  bool alike = average > 0.8 * longest;          // (pieces of tiles are more so than the tiles)
  if (byte && t.batch > 1) {
    average *= 0.6;
    alike = false;
  }
  if (p.f.row_first != nullptr) {
    average = longest / 8.;
    longest /= 3.;
    equal = alike = false;
  }
  ChunkCut best{1, 1, 1, 0.};
  double least = 0.;
  for (int i = 0; i < 3; ++i) {
    const int ks = 1 << i, tiles = chunk_tiles(sh, t.batch, t.n_rows, t.max_new, ks);
    const double rows = kPcRows<1> / ks, page = kPageUs[byte][sh.head_dim == 64][i] * (byte && p.f.cap_in > 0.f ? 1.2 : 1.);
    // of several sequences' last tiles half are empty, on average
    const double likely = t.batch == 1 ? tiles : std::min<double>(tiles, double(t.n_rows) * (sh.n_q_heads / sh.n_kv_heads) / rows + t.batch / 2.);
    for (int splits = 1; splits <= std::min(kPcMaxSplits, t.max_pages); ++splits) {
      if (splits > 1 && size_t(tiles) * sh.n_kv_heads * splits * chunk_piece_bytes(sh, ks) > (byte ? kPcMostPiecesByte : kPcMostPieces) * chunk_piece_bytes(sh, 1)) break;
      const double pieces = likely * sh.n_kv_heads * splits, rounds = pieces / kChipCus;
      double us = std::ceil(longest / splits) * page + item_us;
      us = equal || (splits > 1 && alike) ? std::ceil(rounds) * us
                                          : std::max(us, rounds * (average / splits * page + item_us) + (byte ? 0.3 * us : 0.));
      if (splits > 1) us += 4. + pieces * rows * sh.head_dim * 8. / (byte ? 3e6 : 4e6);
      if ((i == 0 && splits == 1) || us < least) {
        least = us;
        best = ChunkCut{ks, splits, tiles, us};
      }
    }
  }
  return best;
}
// The merge of a call's pieces, where there are several (paged_chunk.hip).
void launch_chunk_merge(int d, int ks, const PagedChunk& c, hipStream_t stream);

}  // namespace actqkv
