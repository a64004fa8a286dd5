// The account of the attention weight after a chunk or a prompt: for every cached token, the sum over rows of exp(score - lse).
//
// A workgroup of 8 wavefronts takes 128 keys (fp32) or 256 (bf16) of one (sequence, KV head) and walks the voting rows, the G heads of
// a row side by side.  S = Q K^T with the rows as the first operand and the keys as the second leaves a lane with scores of ONE
// key, 16 rows of it in its registers: the sum over rows needs no exchange.  A wavefront keeps its keys in registers for the whole
// walk (straight from memory, each byte read once per 4 wavefronts that do not share it) and reads the rows from LDS, 128 at a
// time, double buffered, filled without registers in between; four wavefronts take the first 64 of them, four the others, in two
// blocks of 32: the multiply-adds and exponentials of the first between the products of the second.  Those and an addition per
// score bound it with the products: 2048 rows of each of 2 sequences at 16K tokens, 32 heads, 634 us (813 TFLOP/s); 64 rows a step, a block
// each, 687; 4 wavefronts a workgroup and two workgroups a compute unit 880 (their registers spill); the last 64 rows of 4
// sequences at 8K, 28 heads, 35 us, of which the products are 12: two rounds of the chip, each with its first keys and rows to wait for.
//
// Rows with spans of their own are walked from the first to the last that sees any of the workgroup's keys (documents, as many rows
// and tokens as above at 8192: with the attention 239 us instead of 340).  A cap is the polynomial of the attention's where a wavefront's
// scores are small, a bias two instructions on positions relative to the workgroup's first key.  (With 128 channels in bf16 6 registers are in
// scratch under a cap, 17 with a bias too.)
//
// Where keys alone do not fill the chip, the rows are cut into pieces whose sums a second launch adds up, in order.  Sums of
// 16 rows are added to the running sum, not single terms: its rounding would pass 1e-6 after some thousand.
#include "mfma_util.h"
#include "paged.h"

namespace actqkv {

constexpr int kPwThreads = 512, kPwWaves = kPwThreads / 64;
constexpr int kPwRows = 128;                     // rows (with a head each) of a step
constexpr int kPwWgs = 512;                      // workgroups that a call is cut into

// Keys of a wavefront and of a workgroup; 16-byte operands of a row.
template <typename T, int D> struct PwShape {
  static constexpr int kGroups = sizeof(T) == 2 ? 2 : 1;          // of 32 keys, per wavefront
  static constexpr int kKeys = 4 * 32 * kGroups;
  static constexpr int kRowBytes = D * int(sizeof(T));
  static constexpr int kSteps = kRowBytes / 32;
  static __device__ __forceinline__ uint32_t swizzle(int r) { return kRowBytes == 128 ? (r >> 1) & 7 : r & 15; }
  static __device__ __forceinline__ f32x16 product(const u32x4& a, const u32x4& b, f32x16 c) {
    if constexpr (sizeof(T) == 2) {
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
      return c;
    }
  }
};

struct PagedVotes {
  PagedAttn a;
  PagedWeights w;
  int key_tiles, pieces;
  float* part;               // [pair][piece][key_tiles * kKeys], or NULL: one piece
};

template <typename T, int D, bool kCap, bool kBias>
__device__ __forceinline__ void votes_body(const PagedVotes& c) {
  typedef PwShape<T, D> S;
  constexpr int kG = S::kGroups, kBytes = kPwRows * S::kRowBytes, kPieces = kBytes / 1024 / kPwWaves;
  constexpr int kRowsOf1k = 1024 / S::kRowBytes, kChunks = S::kRowBytes / 16;
  typedef std::conditional_t<sizeof(T) == 2, CapShort, CapForm> Cap;
  __shared__ __attribute__((aligned(16))) char rows_lds[2][kBytes];
  __shared__ __attribute__((aligned(16))) float lse_lds[2][kPwRows], slope_lds[2][kPwRows], ahead_lds[2][kPwRows];
  __shared__ __attribute__((aligned(16))) int lo_lds[2][kPwRows], len_lds[2][kPwRows];
  __shared__ SpanOfRows seen_lds[2][kPwRows / 32];
  __shared__ float sum_lds[S::kKeys];
  const PagedAttn& p = c.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, half = lane >> 5, kg = wave & 3, rh = wave >> 2;
  const int group = p.n_q_heads / p.n_kv_heads;
  const int hk = blockIdx.x % p.n_kv_heads, rest = blockIdx.x / p.n_kv_heads;
  const int piece = rest % c.pieces, tile = rest / c.pieces, s = blockIdx.y;
  const PagedSeq seq = paged_seq(p.t, s);
  const int key0 = tile * S::kKeys, wkey0 = key0 + kg * 32 * kG;  // the workgroup's first key, this wavefront's
  const int w0 = seq.n - seq.m;

  // ---- the rows that vote, of those the ones that can see a key of this tile at all
  int i0 = max(seq.m - c.w.rows, 0), i1 = seq.m;
  if (p.f.row_end == nullptr) i0 = min(max(i0, key0 - w0), seq.m);   // row i sees positions up to w0 + i
  if (p.f.window > 0) i1 = int(min(int64_t(i1), int64_t(key0) + S::kKeys - 1 + p.f.window - w0));
  if (key0 >= seq.n) i1 = i0;
  if ((p.f.row_first != nullptr || p.f.row_end != nullptr) && i1 > i0) {   // of rows with spans of their own from the first to the last that does
    __shared__ int range[2];
    if (tid == 0) {
      range[0] = i1;
      range[1] = i0;
    }
    __syncthreads();
    for (int i = i0 + tid; i < i1; i += kPwThreads) {
      const PagedSpan v = paged_span(p.f, seq.row0 + i, w0 + i, seq.n);
      if (v.hi > max(v.lo, key0) && v.lo < key0 + S::kKeys) {
        atomicMin(&range[0], i);
        atomicMax(&range[1], i + 1);
      }
    }
    __syncthreads();
    i0 = __builtin_amdgcn_readfirstlane(range[0]);
    i1 = __builtin_amdgcn_readfirstlane(range[1]);
  }
  const int f0 = i0 * group, f1 = max(i1, i0) * group;
  const int steps = (f1 - f0 + kPwRows - 1) / kPwRows, per = (steps + c.pieces - 1) / c.pieces;
  const int st0 = piece * per, st1 = min(steps, st0 + per);

  // ---- this wavefront's keys as second operands, and whether their page exists
  const int page_index = wkey0 / kBlock;
  const int page = wkey0 < seq.n && st0 < st1 ? __builtin_amdgcn_readfirstlane(paged_page(p.t, s, page_index)) : -1;
  u32x4 kreg[kG][S::kSteps];
  if (page >= 0) {
    const char* at = static_cast<const char*>(p.k_pages) +
                     ((size_t(page) * p.n_kv_heads + hk) * kBlock + (wkey0 % kBlock) + n) * S::kRowBytes + 16 * half;
#pragma unroll
    for (int gk = 0; gk < kG; ++gk)
#pragma unroll
      for (int j = 0; j < S::kSteps; ++j) kreg[gk][j] = *reinterpret_cast<const u32x4*>(at + gk * 32 * S::kRowBytes + j * 32);
  } else {
#pragma unroll
    for (int gk = 0; gk < kG; ++gk)
#pragma unroll
      for (int j = 0; j < S::kSteps; ++j) kreg[gk][j] = u32x4{0, 0, 0, 0};
  }

  // ---- staging of the rows of a step: their queries into LDS, and by the first two wavefronts what else a row has
  auto fetch = [&](int st, int stage) {
    const int f = f0 + st * kPwRows;
    const int first = f / group;
    const char* base = uniform_ptr(static_cast<const char*>(p.q) +
                                   (size_t(seq.row0 + first) * p.n_q_heads + hk * group) * S::kRowBytes);
    const uint32_t row_stride = uint32_t(p.n_q_heads) * S::kRowBytes;
    const __amdgpu_buffer_rsrc_t src = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, 0x7fffffff, 0x00020000);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int r = (kPieces * wave + i) * kRowsOf1k + lane / kChunks;
      const int fr = min(f + r, f1 - 1), ir = fr / group;          // (rows behind the last repeat it and do not vote)
      const uint32_t off = uint32_t(ir - first) * row_stride + uint32_t(fr - ir * group) * S::kRowBytes +
                           ((uint32_t(lane % kChunks) ^ S::swizzle(r)) << 4);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (__attribute__((address_space(3))) void*)(rows_lds[stage] + (kPieces * wave + i) * 1024),
                                               16, off, 0, 0, 0);
    }
  };
  float my_lse = 0.f, my_slope = 0.f;
  PagedSpan my_span{0x7fffffff, 0};
  float my_ahead = 0.f;                          // its position less the workgroup's first key
  auto row_read = [&](int st) {
    const int f = f0 + st * kPwRows + tid;
    my_span = PagedSpan{0x7fffffff, 0};
    my_lse = my_slope = 0.f;
    my_ahead = 0.f;
    if (f < f1) {
      const int i = f / group, head = hk * group + (f - i * group), row = seq.row0 + i;
      my_lse = p.lse[size_t(row) * p.n_q_heads + head] * kLog2e;
      if (kBias) my_slope = p.f.slopes[head] * kLog2e;
      if (kBias) my_ahead = float(w0 + i - key0);
      const PagedSpan v = paged_span(p.f, row, w0 + i, seq.n);
      if (v.hi > v.lo && my_lse > -INFINITY) my_span = v;
    }
  };
  auto row_write = [&](int stage) {
    lse_lds[stage][tid] = my_span.hi > 0 ? my_lse : 0.f;
    lo_lds[stage][tid] = my_span.lo;
    len_lds[stage][tid] = int(my_span.length());
    if (kBias) {
      slope_lds[stage][tid] = my_slope;
      ahead_lds[stage][tid] = my_ahead;
    }
    const SpanOfRows seen = span_of_rows(my_span);
    if (n == 0) seen_lds[stage][2 * wave + half] = seen;
  };
  float sum[kG], key_at[kG];                     // key_at: this lane's keys, from the workgroup's first on
#pragma unroll
  for (int gk = 0; gk < kG; ++gk) {
    sum[gk] = 0.f;
    key_at[gk] = float(kg * 32 * kG + 32 * gk + n);
  }
  if (st0 < st1) {
    fetch(st0, 0);
    if (wave < kPwRows / 64) {
      row_read(st0);
      row_write(0);
    }
  }
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  // a wavefront's rows of a step: two blocks of 32, whose products and exponentials take turns
  const uint32_t a_off0 = uint32_t(64 * rh + n) * S::kRowBytes + ((uint32_t(half) ^ S::swizzle(n)) << 4);
  for (int st = st0; st < st1; ++st) {
    const int stage = (st - st0) & 1;
    const bool next = st + 1 < st1;
    if (next && wave < kPwRows / 64) row_read(st + 1);
    bool visible[2], masked[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const SpanOfRows seen = seen_lds[stage][2 * rh + b];
      const int lo_any = __builtin_amdgcn_readfirstlane(seen.lo_any), hi_any = __builtin_amdgcn_readfirstlane(seen.hi_any);
      const int lo_all = __builtin_amdgcn_readfirstlane(seen.lo_all), hi_all = __builtin_amdgcn_readfirstlane(seen.hi_all);
      visible[b] = page >= 0 && wkey0 < hi_any && wkey0 + 32 * kG > lo_any;
      masked[b] = wkey0 < lo_all || wkey0 + 32 * kG > hi_all;
    }
    f32x16 acc[2][kG];
    constexpr int kRing = S::kSteps < 8 ? S::kSteps : 8;         // operands on their way
    auto row_operand = [&](int b, int j) {
      return *reinterpret_cast<const u32x4*>(rows_lds[stage] + b * 32 * S::kRowBytes + (a_off0 ^ (uint32_t(j) << 5)));
    };
    // register i is row 64 rh + 32 b + 8 (i / 4) + 4 half + i % 4, the lane's key wkey0 + 32 gk + n
    auto first_row = [&](int b, int q) { return 64 * rh + 32 * b + 8 * q + 4 * half; };
    const float in = kCap ? p.f.cap_in : p.f.scale_log2e;
    Cap cap;
    if constexpr (kCap) {
      if constexpr (sizeof(T) == 2) cap = cap_short(in, p.f.cap_log2e);
      else cap = cap_form(in, p.f.cap_log2e);
    }
    bool small[2];
    auto weights_of = [&](int b, int q) {        // a quarter of a block's
      if constexpr (kCap) {
        if (q == 0) small[b] = cap_is_small(acc[b], in, sizeof(T) == 2 ? kTanhShort : kTanhSmall);
      }
      f32x4 less = *reinterpret_cast<const f32x4*>(&lse_lds[stage][first_row(b, q)]);
      f32x4 slope = {0.f, 0.f, 0.f, 0.f}, ahead = {0.f, 0.f, 0.f, 0.f};
      if constexpr (kBias) {
        slope = *reinterpret_cast<const f32x4*>(&slope_lds[stage][first_row(b, q)]);
        ahead = *reinterpret_cast<const f32x4*>(&ahead_lds[stage][first_row(b, q)]);
      }
      // of a score's exponent what is not the product's: the bias and the sum over the row's keys
      auto rest = [&](int e, int gk) { return kBias ? fmaf(-slope[e], fabsf(ahead[e] - key_at[gk]), -less[e]) : -less[e]; };
      if constexpr (kCap) {
        if (!small[b]) {
#pragma unroll
          for (int gk = 0; gk < kG; ++gk)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              acc[b][gk][4 * q + e] = __builtin_amdgcn_exp2f(paged_tanh(acc[b][gk][4 * q + e] * in, p.f.cap_log2e) + rest(e, gk));
          return;
        }
      }
#pragma unroll
      for (int gk = 0; gk < kG; ++gk)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = acc[b][gk][4 * q + e];
          acc[b][gk][4 * q + e] = __builtin_amdgcn_exp2f(fmaf(x, kCap ? cap.factor(x) : in, rest(e, gk)));
        }
    };
    auto products = [&](int b, bool beside) {    // of block b; beside them the weights of the block before
      u32x4 ring[kRing];
#pragma unroll
      for (int j = 0; j < kRing; ++j) ring[j] = row_operand(b, j);
#pragma unroll
      for (int gk = 0; gk < kG; ++gk)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[b][gk][i] = 0.f;
#pragma unroll
      for (int j = 0; j < S::kSteps; ++j) {
#pragma unroll
        for (int gk = 0; gk < kG; ++gk) acc[b][gk] = S::product(ring[j % kRing], kreg[gk][j], acc[b][gk]);
        if (j + kRing < S::kSteps) ring[j % kRing] = row_operand(b, j + kRing);
        if (beside && j % (S::kSteps / 4) == 0) weights_of(0, j / (S::kSteps / 4));
      }
    };
    auto add = [&](int b) {
      if (masked[b]) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const u32x4 lo = *reinterpret_cast<const u32x4*>(&lo_lds[stage][first_row(b, q)]);
          const u32x4 len = *reinterpret_cast<const u32x4*>(&len_lds[stage][first_row(b, q)]);
#pragma unroll
          for (int gk = 0; gk < kG; ++gk)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              acc[b][gk][4 * q + e] = span_holds(wkey0 + 32 * gk + n - int(lo[e]), len[e]) ? acc[b][gk][4 * q + e] : 0.f;
        }
      }
#pragma unroll
      for (int gk = 0; gk < kG; ++gk) {
        float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 16; ++i) t[i & 3] += acc[b][gk][i];
        sum[gk] += (t[0] + t[1]) + (t[2] + t[3]);
      }
    };
    if (visible[0]) products(0, false);
    if (next) fetch(st + 1, stage ^ 1);
    if (visible[0] && visible[1]) {
      products(1, true);
      add(0);
    } else if (visible[0]) {
#pragma unroll
      for (int q = 0; q < 4; ++q) weights_of(0, q);
      add(0);
    } else if (visible[1]) {
      products(1, false);
    }
    if (visible[1]) {
#pragma unroll
      for (int q = 0; q < 4; ++q) weights_of(1, q);
      add(1);
    }
    if (next && wave < kPwRows / 64) row_write(stage ^ 1);
    __builtin_amdgcn_s_waitcnt(0);               // this wavefront's share of the next rows has landed in LDS
    __syncthreads();
  }
  // ---- the two lanes of a key, then the two sets of rows
#pragma unroll
  for (int gk = 0; gk < kG; ++gk) sum[gk] = lane_pair<32>(sum[gk], [](float x, float y) { return x + y; });
  const int mine = kg * 32 * kG + n;
  if (rh == 1 && half == 0) {
#pragma unroll
    for (int gk = 0; gk < kG; ++gk) sum_lds[mine + 32 * gk] = sum[gk];
  }
  __syncthreads();
  if (rh == 1 || half == 1) return;
  const int pair = s * p.n_kv_heads + hk;
#pragma unroll
  for (int gk = 0; gk < kG; ++gk) {
    const int at = mine + 32 * gk, key = key0 + at;
    const float v = sum[gk] + sum_lds[at];
    if (c.part != nullptr) {
      c.part[(size_t(pair) * c.pieces + piece) * (size_t(c.key_tiles) * S::kKeys) + key] = v;
    } else if (key < p.t.max_pages * kBlock) {
      const size_t to = size_t(pair) * c.w.stride + key;
      c.w.out[to] = c.w.in[to] + v;
    }
  }
}
template <typename T, int D, bool kCap, bool kBias>
__global__ __launch_bounds__(kPwThreads) void paged_votes_kernel(PagedVotes c) {
  votes_body<T, D, kCap, kBias>(c);
}

// weights_out = weights_in + the pieces, in order: a key a thread.
constexpr int kVsThreads = 256;
__global__ __launch_bounds__(kVsThreads) void paged_votes_sum_kernel(PagedVotes c, int keys) {
  const int key = blockIdx.x * kVsThreads + threadIdx.x, pair = blockIdx.y;
  if (key >= c.a.t.max_pages * kBlock) return;
  float v = 0.f;
  for (int i = 0; i < c.pieces; ++i) v += c.part[(size_t(pair) * c.pieces + i) * keys + key];
  const size_t to = size_t(pair) * c.w.stride + key;
  c.w.out[to] = c.w.in[to] + v;
}

// ---- few voting rows: so many (row, query head) pairs of a sequence as LDS holds, staged once.  Every wavefront has 32 keys at a time to
// itself and the next 32 on their way, so that nothing is waited for in common: bound by the reading of the keys.  Attention included, against
// the kernel above: 35 sequences of up to 19 rows at up to 16K tokens, the last 5 rows counting, 622 | 850 us; 43 of up to 12 under a window
// of 338 at 15K 52 | 121 (most keys only have their account copied); 4 x 512 rows at 8K, the last 8, 32 and 64 counting, 207 | 219, 218 | 223, 237 | 236.
constexpr int kPfThreads = 512, kPfWaves = kPfThreads / 64;
constexpr int kPfBytes = 65536;                  // of rows in LDS; two workgroups a compute unit
constexpr int kPfWgs = 1024;                     // workgroups that a call is cut into
template <typename T, int D> constexpr int kPfRows = kPfBytes / PwShape<T, D>::kRowBytes;

template <typename T, int D, bool kCap, bool kBias>
__device__ __forceinline__ void votes_few_body(const PagedVotes& c) {
  typedef PwShape<T, D> S;
  typedef std::conditional_t<sizeof(T) == 2, CapShort, CapForm> Cap;
  constexpr int kRows = kPfRows<T, D>, kRowsOf1k = 1024 / S::kRowBytes, kChunks = S::kRowBytes / 16;
  __shared__ __attribute__((aligned(16))) char rows_lds[kPfBytes];
  __shared__ __attribute__((aligned(16))) float lse_lds[kRows], slope_lds[kBias ? kRows : 4], ahead_lds[kBias ? kRows : 4];
  __shared__ __attribute__((aligned(16))) int lo_lds[kRows], len_lds[kRows];
  __shared__ SpanOfRows seen_lds[kRows / 32];
  const PagedAttn& p = c.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, half = lane >> 5;
  const int group = p.n_q_heads / p.n_kv_heads;
  const int hk = blockIdx.x % p.n_kv_heads, wg = blockIdx.x / p.n_kv_heads, s = blockIdx.y;
  const PagedSeq seq = paged_seq(p.t, s);
  const int w0 = seq.n - seq.m, i0 = max(seq.m - c.w.rows, 0);
  const int f0 = i0 * group, n_pairs = seq.m * group - f0, blocks = (n_pairs + 31) / 32;

  // ---- the rows, once
  if (n_pairs > 0) {
    const char* base = uniform_ptr(static_cast<const char*>(p.q) + (size_t(seq.row0 + i0) * p.n_q_heads + hk * group) * S::kRowBytes);
    const uint32_t row_stride = uint32_t(p.n_q_heads) * S::kRowBytes;
    const __amdgpu_buffer_rsrc_t src = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, 0x7fffffff, 0x00020000);
    for (int piece = wave; piece * kRowsOf1k < blocks * 32; piece += kPfWaves) {
      const int r = piece * kRowsOf1k + lane / kChunks, fr = min(r, n_pairs - 1), ir = fr / group;   // (rows behind the last repeat it and do not vote)
      const uint32_t off = uint32_t(ir) * row_stride + uint32_t(fr - ir * group) * S::kRowBytes +
                           ((uint32_t(lane % kChunks) ^ S::swizzle(r)) << 4);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (__attribute__((address_space(3))) void*)(rows_lds + piece * 1024), 16, off, 0, 0, 0);
    }
    for (int r0 = wave * 64; r0 < blocks * 32; r0 += kPfThreads) {
      const int r = r0 + lane;
      PagedSpan span{0x7fffffff, 0};
      float lse = 0.f;
      if (r < n_pairs) {
        const int i = i0 + r / group, head = hk * group + r % group, row = seq.row0 + i;
        const PagedSpan v = paged_span(p.f, row, w0 + i, seq.n);
        const float l = p.lse[size_t(row) * p.n_q_heads + head] * kLog2e;
        if (v.hi > v.lo && l > -INFINITY) {
          span = v;
          lse = l;
        }
        if constexpr (kBias) {
          slope_lds[r] = p.f.slopes[head] * kLog2e;
          ahead_lds[r] = float(i);
        }
      } else if (kBias && r < blocks * 32) {
        slope_lds[r] = ahead_lds[r] = 0.f;
      }
      const SpanOfRows seen = span_of_rows(span);
      if (r < blocks * 32) {
        lse_lds[r] = lse;
        lo_lds[r] = span.lo;
        len_lds[r] = int(span.length());
        if (n == 0) seen_lds[r / 32] = seen;
      }
    }
  }
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  int lo_any = 0x7fffffff, hi_any = 0;           // what any of them sees
  for (int b = 0; b < blocks; ++b) {
    lo_any = min(lo_any, seen_lds[b].lo_any);
    hi_any = max(hi_any, seen_lds[b].hi_any);
  }
  lo_any = __builtin_amdgcn_readfirstlane(lo_any);
  hi_any = __builtin_amdgcn_readfirstlane(hi_any);

  const int groups = p.t.max_pages * (kBlock / 32), stride = c.key_tiles * kPfWaves;   // (key_tiles: workgroups of a sequence and KV head)
  const size_t out_row = size_t(s * p.n_kv_heads + hk) * c.w.stride;
  const char* kp = static_cast<const char*>(p.k_pages);
  int my_page = -1;
  auto page_at = [&](int k, int g) {             // the page of key group g, this wavefront's k-th, of those that somebody sees; -1: none
    if ((k & 63) == 0) {
      const int mine = g + lane * stride, key = mine * 32;
      my_page = mine < groups && key < hi_any && key + 32 > lo_any ? paged_page(p.t, s, key / kBlock) : -1;
    }
    return __builtin_amdgcn_readlane(my_page, k & 63);
  };
  auto load = [&](u32x4 (&to)[S::kSteps], int page, int g) {
    if (page < 0) return;
    const char* at = kp + ((size_t(page) * p.n_kv_heads + hk) * kBlock + (g * 32) % kBlock + n) * S::kRowBytes + 16 * half;
#pragma unroll
    for (int j = 0; j < S::kSteps; ++j) to[j] = *reinterpret_cast<const u32x4*>(at + j * 32);
  };
  const float in = kCap ? p.f.cap_in : p.f.scale_log2e;
  Cap cap;
  if constexpr (kCap) {
    if constexpr (sizeof(T) == 2) cap = cap_short(in, p.f.cap_log2e);
    else cap = cap_form(in, p.f.cap_log2e);
  }
  const uint32_t a_off0 = uint32_t(n) * S::kRowBytes + ((uint32_t(half) ^ S::swizzle(n)) << 4);
  auto process = [&](const u32x4 (&keys)[S::kSteps], int page, int g) {
    const int key0 = g * 32;
    if (page < 0 && c.w.in == c.w.out) return;
    const float before = half == 0 ? c.w.in[out_row + key0 + n] : 0.f;
    float sum = 0.f;
    if (page >= 0) {
      const float at = float(key0 + n - w0);
      for (int b = 0; b < blocks; ++b) {
        const SpanOfRows seen = seen_lds[b];
        if (key0 >= __builtin_amdgcn_readfirstlane(seen.hi_any) || key0 + 32 <= __builtin_amdgcn_readfirstlane(seen.lo_any)) continue;
        const bool masked = key0 < __builtin_amdgcn_readfirstlane(seen.lo_all) || key0 + 32 > __builtin_amdgcn_readfirstlane(seen.hi_all);
        f32x16 acc[1];
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[0][i] = 0.f;
#pragma unroll
        for (int j = 0; j < S::kSteps; ++j)
          acc[0] = S::product(*reinterpret_cast<const u32x4*>(rows_lds + b * 32 * S::kRowBytes + (a_off0 ^ (uint32_t(j) << 5))), keys[j], acc[0]);
        bool small = true;
        if constexpr (kCap) small = cap_is_small(acc, in, sizeof(T) == 2 ? kTanhShort : kTanhSmall);
        float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 0; q < 4; ++q) {            // register 4 q + e is row 32 b + 8 q + 4 half + e
          const int r = 32 * b + 8 * q + 4 * half;
          const f32x4 less = *reinterpret_cast<const f32x4*>(&lse_lds[r]);
          f32x4 slope = {0.f, 0.f, 0.f, 0.f}, ahead = {0.f, 0.f, 0.f, 0.f};
          if constexpr (kBias) {
            slope = *reinterpret_cast<const f32x4*>(&slope_lds[r]);
            ahead = *reinterpret_cast<const f32x4*>(&ahead_lds[r]);
          }
          float w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = acc[0][4 * q + e], rest = kBias ? fmaf(-slope[e], fabsf(ahead[e] - at), -less[e]) : -less[e];
            if constexpr (kCap) w[e] = small ? fmaf(x, cap.factor(x), rest) : paged_tanh(x * in, p.f.cap_log2e) + rest;
            else w[e] = fmaf(x, in, rest);
            w[e] = __builtin_amdgcn_exp2f(w[e]);
          }
          if (masked) {
            const u32x4 lo = *reinterpret_cast<const u32x4*>(&lo_lds[r]), len = *reinterpret_cast<const u32x4*>(&len_lds[r]);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = span_holds(key0 + n - int(lo[e]), len[e]) ? w[e] : 0.f;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) t[e] += w[e];
        }
        sum += (t[0] + t[1]) + (t[2] + t[3]);
      }
      sum = lane_pair<32>(sum, [](float x, float y) { return x + y; });
    }
    if (half == 0) c.w.out[out_row + key0 + n] = before + sum;
  };
  u32x4 ka[S::kSteps], kb[S::kSteps];
  int g = wg * kPfWaves + wave;
  if (g >= groups) return;
  int pa = page_at(0, g);
  load(ka, pa, g);
  for (int k = 0; g < groups; k += 2, g += 2 * stride) {
    const int pb = g + stride < groups ? page_at(k + 1, g + stride) : -1;
    load(kb, pb, g + stride);
    process(ka, pa, g);
    if (g + stride >= groups) break;
    pa = g + 2 * stride < groups ? page_at(k + 2, g + 2 * stride) : -1;
    load(ka, pa, g + 2 * stride);
    process(kb, pb, g + stride);
  }
}
template <typename T, int D, bool kCap, bool kBias>
__global__ __launch_bounds__(kPfThreads) void paged_votes_few_kernel(PagedVotes c) {
  votes_few_body<T, D, kCap, kBias>(c);
}

// ---- host side
static int votes_keys(const actqkv_shape& sh) { return sh.dtype == ACTQKV_F32 ? PwShape<float, 64>::kKeys : PwShape<uint16_t, 64>::kKeys; }

// Pieces hold kPwWgs workgroups' sums and, rounded up, as many again.
size_t paged_votes_scratch_most(const actqkv_shape& sh) { return size_t(2 * kPwWgs) * votes_keys(sh) * sizeof(float); }

template <typename T, int D>
static void launch_votes(const PagedVotes& c, hipStream_t stream) {
  const bool cap = c.a.f.cap_in > 0.f, bias = c.a.f.slopes != nullptr;
  const dim3 grid(unsigned(c.a.n_kv_heads) * c.key_tiles * c.pieces, c.a.t.batch);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kPwThreads), 0, stream, c); };
  if (cap && bias) launch(paged_votes_kernel<T, D, true, true>);
  else if (cap) launch(paged_votes_kernel<T, D, true, false>);
  else if (bias) launch(paged_votes_kernel<T, D, false, true>);
  else launch(paged_votes_kernel<T, D, false, false>);
}

template <typename T, int D>
static bool launch_votes_few(PagedVotes c, hipStream_t stream) {
  const int group = c.a.n_q_heads / c.a.n_kv_heads;
  if (int64_t(std::min(c.w.rows, c.a.t.max_new)) * group > kPfRows<T, D>) return false;
  const bool cap = c.a.f.cap_in > 0.f, bias = c.a.f.slopes != nullptr;
  const int64_t pairs = int64_t(c.a.n_kv_heads) * c.a.t.batch;
  c.key_tiles = int(std::min<int64_t>((c.a.t.max_pages * int64_t(kBlock / 32) + kPfWaves - 1) / kPfWaves, (kPfWgs + pairs - 1) / pairs));
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(unsigned(c.a.n_kv_heads) * c.key_tiles, c.a.t.batch), dim3(kPfThreads), 0, stream, c);
  };
  if (cap && bias) launch(paged_votes_few_kernel<T, D, true, true>);
  else if (cap) launch(paged_votes_few_kernel<T, D, true, false>);
  else if (bias) launch(paged_votes_few_kernel<T, D, false, true>);
  else launch(paged_votes_few_kernel<T, D, false, false>);
  return true;
}

int launch_paged_votes(const actqkv_shape& sh, const PagedAttn& p, const PagedWeights& w, const Workspace& ws, hipStream_t stream) {
  PagedVotes c;
  c.a = p;
  c.w = w;
  c.pieces = 1;
  c.part = nullptr;
  const bool few = sh.dtype == ACTQKV_F32 ? (sh.head_dim == 64 ? launch_votes_few<float, 64>(c, stream) : launch_votes_few<float, 128>(c, stream))
                                          : (sh.head_dim == 64 ? launch_votes_few<uint16_t, 64>(c, stream) : launch_votes_few<uint16_t, 128>(c, stream));
  if (few) return hip_status("paged attention weights");
  const int keys = votes_keys(sh);
  c.key_tiles = (p.t.max_pages * kBlock + keys - 1) / keys;
  const int64_t items = int64_t(c.key_tiles) * p.n_kv_heads * p.t.batch;
  const int64_t steps = (int64_t(std::min(w.rows, p.t.max_new)) * (sh.n_q_heads / sh.n_kv_heads) + kPwRows - 1) / kPwRows;
  c.pieces = int(std::max<int64_t>(1, std::min((kPwWgs + items - 1) / items, steps)));
  c.part = c.pieces > 1 ? ws.scratch_f32() : nullptr;
  if (sh.dtype == ACTQKV_F32) {
    if (sh.head_dim == 64) launch_votes<float, 64>(c, stream);
    else launch_votes<float, 128>(c, stream);
  } else {
    if (sh.head_dim == 64) launch_votes<uint16_t, 64>(c, stream);
    else launch_votes<uint16_t, 128>(c, stream);
  }
  if (c.pieces > 1) {
    const dim3 grid((p.t.max_pages * kBlock + kVsThreads - 1) / kVsThreads, p.n_kv_heads * p.t.batch);
    hipLaunchKernelGGL(paged_votes_sum_kernel, grid, dim3(kVsThreads), 0, stream, c, c.key_tiles * keys);
  }
  return hip_status("paged attention weights");
}

}  // namespace actqkv
