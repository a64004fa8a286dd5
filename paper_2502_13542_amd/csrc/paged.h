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

// The sequence that query tile `tile` of rows_per rows belongs to, and the tile's number in it (from its last rows on: they see
// the most keys and start first); false behind the last one.
__device__ __forceinline__ bool paged_find_tile(const PagedTable& t, int tile, int group, int rows_per, int& s, int& local) {
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < t.batch; s0 += 64) {
    int n = 0;
    if (s0 + lane < t.batch) {
      const PagedSeq q = paged_seq(t, s0 + lane);
      n = (q.m * group + rows_per - 1) / rows_per;
    }
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
};
__device__ __forceinline__ PagedSpan paged_span(const PagedForm& f, int row, int pos, int n) {
  PagedSpan v{0, 0};
  if (pos < 0) return v;                         // more rows than tokens: the row is not in the cache
  v.hi = f.row_end != nullptr ? min(f.row_end[row], n) : pos + 1;
  if (f.row_first != nullptr) v.lo = max(f.row_first[row], 0);
  if (f.window > 0) v.lo = max(v.lo, pos - f.window + 1);
  return v;
}

// tanh to 2 units of the last place: below 0.625 x + x^3 times a polynomial in x^2 (least squares, 4e-9 of it), above
// 1 - 2 / (e^2x + 1).  (That alone loses, by 1 - 1, as many bits as x is small, and a cap multiplies what is lost: scores of
// 3 under a cap of 50 would be off by 6e-6.)
__device__ __forceinline__ float paged_tanh(float x) {
  const float u = x * x;
  float g = fmaf(u, -0.00570404f, 0.02063786f);
  g = fmaf(u, g, -0.05373916f);
  g = fmaf(u, g, 0.13331432f);
  g = fmaf(u, g, -0.33333281f);
  const float small = fmaf(x, u * g, x);
  const float e = __builtin_amdgcn_exp2f(fabsf(x) * (2.f * kLog2e));
  const float large = copysignf(1.f - 2.f * __builtin_amdgcn_rcpf(e + 1.f), x);
  return fabsf(x) < 0.625f ? small : large;
}
// The score, in units of log2, from a product of query and key: far = |position of the query - position of the key|, slope in
// units of log2.
template <bool kCap, bool kBias>
__device__ __forceinline__ float paged_score(const PagedForm& f, float product, float slope, int far) {
  float v = kCap ? f.cap_log2e * paged_tanh(product * f.cap_in) : product * f.scale_log2e;
  if (kBias) v = fmaf(-slope, float(far), v);
  return v;
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
};
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
size_t paged_chunk_scratch_most(const actqkv_shape& sh, int batch, int n_rows, int max_new, int max_pages);
int launch_paged_chunk(const actqkv_shape& sh, const PagedAttn& p, const Workspace& ws, hipStream_t stream);
size_t paged_chunk_f32_scratch_most(const actqkv_shape& sh, int batch, int n_rows, int max_new, int max_pages);
int launch_paged_chunk_f32(const actqkv_shape& sh, const PagedAttn& p, const Workspace& ws, hipStream_t stream);
size_t paged_votes_scratch_most(const actqkv_shape& sh);
int launch_paged_votes(const actqkv_shape& sh, const PagedAttn& p, const PagedWeights& w, const Workspace& ws, hipStream_t stream);
int launch_paged_append(const actqkv_shape& sh, const PagedTable& t, const void* k_new, const void* v_new,
                        void* k_pages, void* v_pages, hipStream_t stream);
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
