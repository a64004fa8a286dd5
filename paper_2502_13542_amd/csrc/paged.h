// The paged cache: what its calls share on the host and on the device.
//
// A page is a cache block: 128 tokens, keys [Hk][128][D], values transposed [Hk][D][128].  Sequence s of a call holds
// its tokens [128 i, 128 i + 128) in page pages[s][i]; its new rows are row_start[s] .. row_start[s + 1] - 1 of q (or
// k_new, v_new), the last of its n_ctx[s] tokens.
#pragma once

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "launch.h"

namespace actqkv {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kMaxPagedRows = 1 << 22;   // rows of a call

struct PagedTable {
  const int32_t* row_start;  // [batch + 1], or NULL: no rows (eviction)
  const int32_t* n_ctx;      // [batch]
  const int32_t* pages;      // [batch][max_pages]
  int batch, n_rows, max_new, max_pages, n_pages;
  int few;                   // (row, query head) pairs of a KV head up to which a sequence is a step kernel's and no other's; 0: none is
};

// Rows and tokens of a sequence, clamped so that no value on the device leads out of an array.
struct PagedSeq {
  int row0, m, n;            // first row, rows, tokens in all (the rows' own included)
};
__device__ __forceinline__ int paged_tokens(const PagedTable& t, int s) {
  return min(max(t.n_ctx[s], 0), t.max_pages * kBlock);
}
__device__ __forceinline__ PagedSeq paged_seq(const PagedTable& t, int s) {
  PagedSeq q;
  q.row0 = min(max(t.row_start[s], 0), t.n_rows);
  q.m = min(min(max(t.row_start[s + 1], q.row0), t.n_rows) - q.row0, t.max_new);
  q.n = paged_tokens(t, s);
  return q;
}
// Page of a sequence's tokens [128 i, 128 i + 128), or -1.
__device__ __forceinline__ int paged_page(const PagedTable& t, int s, int i) {
  const int page = t.pages[size_t(s) * t.max_pages + i];
  return page >= 0 && page < t.n_pages ? page : -1;
}

// Of 64 lanes' counts the inclusive sums.
__device__ __forceinline__ int wave_scan(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int below = __shfl_up(v, d, 64);
    if (lane >= d) v += below;
  }
  return v;
}

// Of 64 lanes' counts the inclusive sums, by the data-parallel primitives.
template <int kCtrl, int kRows>
__device__ __forceinline__ int dpp_add(int v) { return v + __builtin_amdgcn_update_dpp(0, v, kCtrl, kRows, 0xF, false); }
__device__ __forceinline__ int lane_sums(int v) {
  v = dpp_add<0x111, 0xF>(v);                    // row_shr 1, 2, 4, 8
  v = dpp_add<0x112, 0xF>(v);
  v = dpp_add<0x114, 0xF>(v);
  v = dpp_add<0x118, 0xF>(v);
  v = dpp_add<0x142, 0xA>(v);                    // row_bcast 15 into rows 1, 3, then 31 into rows 2, 3
  return dpp_add<0x143, 0xC>(v);
}
// The least and the largest over each half of the lanes, by the data-parallel primitives (through LDS, as a shuffle, a step is 60 ns).
__device__ __forceinline__ int half_min(int v) {
  v = min(v, int(lane_xor32<1>(uint32_t(v))));
  v = min(v, int(lane_xor32<2>(uint32_t(v))));
  v = min(v, int(lane_xor32<4>(uint32_t(v))));
  v = min(v, int(lane_xor32<8>(uint32_t(v))));
  return min(v, int(lane_xor32<16>(uint32_t(v))));
}
__device__ __forceinline__ int half_max(int v) { return ~half_min(~v); }
// What 32 rows see: any of them [lo_any, hi_any), all of them [lo_all, hi_all).
struct SpanOfRows {
  int lo_any, hi_any, lo_all, hi_all;
};

// Query tiles of a sequence.
__device__ __forceinline__ int paged_tiles(const PagedTable& t, const PagedSeq& q, int group, int rows_per) {
  return q.m * group > t.few ? (q.m * group + rows_per - 1) / rows_per : 0;
}
// The sequence that query tile `tile` belongs to, and the tile's number in it (from its last rows on: they see the most keys
// and start first); false behind the last one.
__device__ __forceinline__ bool paged_find_tile(const PagedTable& t, int tile, int group, int rows_per, int& s, int& local) {
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < t.batch; s0 += 64) {
    const int n = s0 + lane < t.batch ? paged_tiles(t, paged_seq(t, s0 + lane), group, rows_per) : 0;
    const int sum = wave_scan(n);
    const unsigned long long mine = __ballot(tile < sum);
    if (mine != 0) {
      const int at = __ffsll(mine) - 1;
      const int end = __builtin_amdgcn_readlane(sum, at);
      s = s0 + at;
      local = end - 1 - tile;
      return true;
    }
    tile -= __builtin_amdgcn_readlane(sum, 63);
  }
  return false;
}

// The sequence that brings row `row`, or -1 (the same in all lanes).
__device__ __forceinline__ int paged_seq_of_row(const PagedTable& t, int row) {
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < t.batch; s0 += 64) {
    bool mine = false;
    if (s0 + lane < t.batch) {
      const PagedSeq q = paged_seq(t, s0 + lane);
      mine = row >= q.row0 && row < q.row0 + q.m;
    }
    const unsigned long long any = __ballot(mine);
    if (any != 0) return s0 + __ffsll(any) - 1;
  }
  return -1;
}

// How scores are formed and which keys a row sees.
struct PagedForm {
  const int32_t* row_first;  // [n_rows] or NULL
  const int32_t* row_end;    // [n_rows] or NULL
  const float* slopes;       // [H] or NULL
  int window;                // 0: none
  float scale_log2e;         // score in units of log2 = product * scale_log2e ...
  float cap_in, cap_log2e;   // ... or cap_log2e * tanh(product * cap_in)
};
// Positions [lo, hi) that a row at position pos of a sequence of n tokens sees (hi <= lo: none).
struct PagedSpan {
  int lo, hi;
  // one comparison a key, unsigned: a second one costs scalar registers for its mask, which 32 of them do not have.  (Neither
  // bound is negative, so that their difference fits.)
  __device__ __forceinline__ uint32_t length() const { return uint32_t(max(hi - lo, 0)); }
};
__device__ __forceinline__ bool span_holds(int key_less_lo, uint32_t length) { return uint32_t(key_less_lo) < length; }
__device__ __forceinline__ PagedSpan paged_span(const PagedForm& f, int row, int pos, int n) {
  PagedSpan v{0, 0};
  if (pos < 0) return v;                         // more rows than tokens: the row is not in the cache
  v.hi = f.row_end != nullptr ? max(min(f.row_end[row], n), 0) : pos + 1;
  if (f.row_first != nullptr) v.lo = max(f.row_first[row], 0);
  if (f.window > 0) v.lo = max(v.lo, pos - f.window + 1);
  return v;
}

// tanh to 2 units of the last place: up to 0.3 x + x^3 times a polynomial in x^2 (least squares, 1.3e-8 of it), above it
// 1 - 2 / (e^2x + 1).  (That alone loses, by 1 - 1, as many bits as x is small, and a cap multiplies what is lost: scores of
// 3 under a cap of 50 would be off by 6e-6.)
constexpr float kTanhSmall = 0.3f;
// A capped score, out * tanh(in * x), as x (b0 + u (b1 + u (b2 + u b3))), u = x x, of a product x in the polynomial's range;
// or x itself, of a score that was capped already.
struct CapForm {
  float b0, b1, b2, b3;
  __device__ __forceinline__ float factor(float x) const {
    const float u = x * x;
    return fmaf(u, fmaf(u, fmaf(u, b3, b2), b1), b0);
  }
};
__device__ __forceinline__ CapForm cap_form(float in, float out) {
  const float b = in * out, k = in * in;
  return CapForm{b, -0.333330558f * b * k, 0.133146743f * b * k * k, -0.0503546844f * b * k * k * k};
}
// The same with a term less, up to 0.2 (1.3e-7 of it): for bf16 storage, where it is an instruction a score in a loop that vector
// instructions bound.
constexpr float kTanhShort = 0.2f;
struct CapShort {
  float b0, b1, b2;
  __device__ __forceinline__ float factor(float x) const {
    const float u = x * x;
    return fmaf(u, fmaf(u, b2, b1), b0);
  }
};
__device__ __forceinline__ CapShort cap_short(float in, float out) {
  const float b = in * out, k = in * in;
  return CapShort{b, -0.33329646f * b * k, 0.1303653f * b * k * k};
}
__device__ __forceinline__ float paged_tanh(float x, float scale) {
  const float e = __builtin_amdgcn_exp2f(fabsf(x) * (2.f * kLog2e));
  float large = copysignf(fmaf(-2.f, __builtin_amdgcn_rcpf(e + 1.f), 1.f), x) * scale;
  asm volatile("" : "+v"(large));                // (a select, not 64 branches)
  return fabsf(x) <= kTanhSmall ? x * cap_form(1.f, scale).factor(x) : large;
}
// The score, in units of log2, from a product of query and key: far = |position of the query - position of the key|, slope in
// units of log2.
template <bool kCap, bool kBias>
__device__ __forceinline__ float paged_score(const PagedForm& f, float product, float slope, int far) {
  float v = kCap ? paged_tanh(product * f.cap_in, f.cap_log2e) : product * f.scale_log2e;
  if (kBias) v = fmaf(-slope, float(far), v);
  return v;
}
// Whether the arguments in * x of a lane's registers, of all lanes, are in the polynomial's range: most of the time, and then a
// cap is 5 instructions a score, otherwise 17.  Said to be the same for the wavefront: from
// a branch that might not be, the two ways' 64 scores come to lie beside each other, in scratch (2 x 2048 rows at 8192 tokens with cap and
// slopes 2120 us instead of 564).  (in^6 has to be a number, too: under a cap of thousands, or of millionths, none is small.)
template <int N>
__device__ __forceinline__ bool cap_is_small(const f32x16 (&x)[N], float in, float most) {
  float mx = 0.f;
#pragma unroll
  for (int g = 0; g < N; ++g)
#pragma unroll
    for (int i = 0; i < 16; i += 2) mx = fmaxf(fmaxf(fabsf(x[g][i]), fabsf(x[g][i + 1])), mx);
  return __builtin_amdgcn_readfirstlane(int(in >= 1e-5f) & int(in <= 1e5f) & int(__all(mx * in <= most))) != 0;
}
// Their scores.  `ahead`: the query's position less that of the key that off(g, i) = 0 would be of.  `cap`, up to `most` of the
// argument: the polynomial.
template <bool kCap, bool kBias, typename Cap, int N, typename Off>
__device__ __forceinline__ void paged_scores(const PagedForm& f, f32x16 (&x)[N], float in, const Cap& cap, float most, float slope,
                                             float ahead, Off off) {
  auto bias = [&](int g, int i) { return kBias ? -slope * fabsf(ahead - float(off(g, i))) : 0.f; };
  if constexpr (kCap) {
    if (cap_is_small(x, in, most)) {
      if (kBias) asm volatile("" : "+v"(ahead));           // (what both branches take of it is not to be taken before them, into 64 registers)
#pragma unroll
      for (int g = 0; g < N; ++g)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[g][i] = fmaf(x[g][i], cap.factor(x[g][i]), bias(g, i));
    } else {
      if (kBias) asm volatile("" : "+v"(ahead));
#pragma unroll
      for (int g = 0; g < N; ++g)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          x[g][i] = paged_tanh(x[g][i] * in, f.cap_log2e) + bias(g, i);
          if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // (of more at once the two ways of tanh take registers that there are not)
        }
    }
  } else {
#pragma unroll
    for (int g = 0; g < N; ++g)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[g][i] = fmaf(x[g][i], in, bias(g, i));
  }
}

struct PagedAttn {
  PagedTable t;
  PagedForm f;
  int n_q_heads, n_kv_heads;
  const void* q;             // [n_rows][H][D]
  const void* k_pages;
  const void* v_pages;
  void* out;                 // [n_rows][H][D]
  float* lse;                // [n_rows][H] or NULL
  const float* k_scales;     // [n_pages][Hk], of pages in 8 bits
  const float* v_scales;
};
__device__ __forceinline__ SpanOfRows span_of_rows(const PagedSpan& v) {
  return SpanOfRows{half_min(v.lo), half_max(v.hi), half_max(v.lo), half_min(v.hi)};
}
struct PagedWeights {
  int rows;                  // the last so many rows of a sequence count
  const float* in;           // [batch][Hk][stride]
  float* out;
  int64_t stride;
};

constexpr int kStepWgs = 1024;            // workgroups that a step call is cut into
bool paged_step_supported(const actqkv_shape& sh, int max_new);
size_t paged_step_scratch_most(const actqkv_shape& sh, int batch, int max_new, int max_pages);
int launch_paged_step(const actqkv_shape& sh, const PagedAttn& p, const PagedWeights* weights, const Workspace& ws,
                      hipStream_t stream);
int launch_paged8_chunk(const actqkv_shape& sh, const PagedAttn& p, const Workspace& ws, hipStream_t stream);
int launch_paged8_chunk_f32(const actqkv_shape& sh, const PagedAttn& p, const Workspace& ws, hipStream_t stream);
size_t paged8_step_scratch_most(const actqkv_shape& sh, int batch);
int launch_paged8_step(const actqkv_shape& sh, const PagedAttn& p, const Workspace& ws, hipStream_t stream);
size_t paged_selected_scratch_most(const actqkv_shape& sh, int batch, int n_rows, int max_new, int max_pages);
int launch_paged_selected(const actqkv_shape& sh, const PagedAttn& p, const int32_t* idx, const int32_t* n_sel, int k_sel,
                          const Workspace& ws, hipStream_t stream);
// (byte: of pages in 8 bits, whose calls are cut into more pieces)
size_t paged_chunk_scratch_most(const actqkv_shape& sh, int batch, int n_rows, int max_new, int max_pages, bool byte);
int launch_paged_chunk(const actqkv_shape& sh, const PagedAttn& p, const Workspace& ws, hipStream_t stream);
size_t paged_chunk_f32_scratch_most(const actqkv_shape& sh, int batch, int n_rows, int max_new, int max_pages, bool byte);
int launch_paged_chunk_f32(const actqkv_shape& sh, const PagedAttn& p, const Workspace& ws, hipStream_t stream);
size_t paged_votes_scratch_most(const actqkv_shape& sh);
int launch_paged_votes(const actqkv_shape& sh, const PagedAttn& p, const PagedWeights& w, const Workspace& ws, hipStream_t stream);
int launch_paged_append(const actqkv_shape& sh, const PagedTable& t, const void* k_new, const void* v_new,
                        void* k_pages, void* v_pages, hipStream_t stream);
// How a call is cut up: cut[0 .. 2] as of actqkv_paged_cut.
void paged_chunk_cut(const actqkv_shape& sh, const PagedAttn& p, int32_t* cut);
void paged_chunk_f32_cut(const actqkv_shape& sh, const PagedAttn& p, int32_t* cut);
void paged_select_cut(const actqkv_shape& sh, const PagedTable& t, int32_t* cut);
bool paged_selected_by_chunks(const actqkv_shape& sh, const PagedAttn& p, int k_sel);
void paged_append_rotated_cut(const actqkv_shape& sh, const PagedTable& t, int32_t* cut);
void paged_append_quantised_cut(const actqkv_shape& sh, const PagedTable& t, bool queries, int32_t* cut);
// Rotation of keys and queries by their position (paged_rotate.h).
struct PagedRotation {
  const float* table;        // [n_positions][2][dims / 2]: cosines, sines; NULL: none (dims 0)
  int n_positions, dims;
  bool interleaved;
  const int32_t* row_pos;    // [n_rows] or NULL: the rows' own positions
};
int launch_paged_append_rotated(const actqkv_shape& sh, const PagedTable& t, const PagedRotation& r, const void* q, const void* k_new,
                                const void* v_new, void* k_pages, void* v_pages, void* q_out, hipStream_t stream);
int launch_paged_append_quantised(const actqkv_shape& sh, const PagedTable& t, const PagedRotation& r, const void* q, const void* k_new,
                             const void* v_new, uint8_t* k_pages, uint8_t* v_pages, float* k_scales, float* v_scales, void* q_out,
                             hipStream_t stream);
int launch_paged_bounds(const actqkv_shape& sh, const PagedTable& t, const void* k_pages, void* bounds, hipStream_t stream);
int launch_paged_select(const actqkv_shape& sh, const PagedTable& t, const void* q, const void* bounds, int k_sel, int keep_first,
                        int keep_last, float* scores, int64_t stride, int32_t* idx, int32_t* n_sel, const Workspace& ws,
                        hipStream_t stream);
struct PagedEvict {
  PagedTable t;
  void* k_pages;
  void* v_pages;
  const float* weights;      // [batch][Hk][stride]
  int64_t stride;
  int keep_first, keep_last, budget;
  const int32_t* to_pages;   // [batch][to_max_pages]; the table itself: in place
  int to_max_pages;
  float* to_weights;         // [batch][Hk][to_stride] or NULL
  int64_t to_stride;
  int32_t* kept;             // [batch][Hk][budget]
  int32_t* n_kept;           // [batch]
  int n_kv_heads;
};
int launch_paged_evict(const actqkv_shape& sh, const PagedEvict& e, hipStream_t stream);

}  // namespace actqkv
