// C ABI of the paged cache: host-side argument checks, then the launchers.
#include <cmath>

#include "checks.h"
#include "paged.h"

namespace actqkv {

// Which kernels a call takes: few rows per sequence or chunks, by the storage type; the votes behind them.
static int launch_paged_attention(const actqkv_shape& sh, PagedAttn p, const PagedWeights* weights, const Workspace& ws,
                                  hipStream_t stream) {
  if (paged_step_supported(sh, p.t.max_new)) return launch_paged_step(sh, p, weights, ws, stream);
  // Sequences of a batch that bring few rows go through the step kernel, in a launch of their own of about 15 us, if they may
  // be so many that their pages, read for a query tile each, would take longer (2 us a page and workgroup).
  const int group = sh.n_q_heads / sh.n_kv_heads, few_rows = 16 / group;
  const int64_t more = std::max<int64_t>(0, int64_t(p.t.n_rows) - int64_t(p.t.batch) * few_rows);
  const int64_t few_most = p.t.batch - (more + p.t.max_new - 1) / p.t.max_new;
  if (few_most * p.t.max_pages * sh.n_kv_heads * 2 > int64_t(20) * kChipCus) {
    ACTQKV_TRY(launch_paged_step(sh, p, nullptr, ws, stream));
    p.t.few = 16;
  }
  ACTQKV_TRY(sh.dtype == ACTQKV_F32 ? launch_paged_chunk_f32(sh, p, ws, stream) : launch_paged_chunk(sh, p, ws, stream));
  return weights != nullptr ? launch_paged_votes(sh, p, *weights, ws, stream) : ACTQKV_OK;
}
// Enough for every call of at most these sizes: of few rows a sequence, none of them takes the chunks' kernels.
static size_t paged_workspace_bytes(const actqkv_shape& sh, int batch, int n_rows, int max_new, int max_pages) {
  size_t most = paged_step_scratch_most(sh, batch, max_new, max_pages);
  if (!paged_step_supported(sh, max_new))
    most = std::max({most, paged_votes_scratch_most(sh),
                     sh.dtype == ACTQKV_F32 ? paged_chunk_f32_scratch_most(sh, batch, n_rows, max_new, max_pages)
                                            : paged_chunk_scratch_most(sh, batch, n_rows, max_new, max_pages)});
  return kCounterBytes + align_up(most, 256);
}

constexpr int kMaxPages = (1 << 30) / kBlock;     // 2^30 tokens: of a sequence, and in the pool
// Caps: their reciprocal is a number, and no capped score is below what the kernels take for a hidden one.
constexpr float kLeastCap = 1e-6f, kLargestCap = 1e6f;

static int check_table(const actqkv_shape* shape, int batch, const int32_t* n_ctx, const int32_t* pages, int max_pages,
                       const void* k_pages, const void* v_pages, int n_pages) {
  ACTQKV_TRY(check_shape(shape));
  ACTQKV_TRY(check_batch(batch));
  if (max_pages < 1 || n_pages < 1)
    return set_error(ACTQKV_EINVAL, "max_pages %d or n_pages %d < 1", max_pages, n_pages);
  if (max_pages > kMaxPages || n_pages > kMaxPages)
    return set_error(ACTQKV_ESHAPE, "max_pages %d or n_pages %d > %d", max_pages, n_pages, kMaxPages);
  ACTQKV_REQUIRE_SMALL(n_ctx, 4);
  ACTQKV_REQUIRE_SMALL(pages, 4);
  ACTQKV_REQUIRE_PTR(k_pages);
  ACTQKV_REQUIRE_PTR(v_pages);
  return ACTQKV_OK;
}

static int check_rows(int n_rows, int max_new) {
  if (n_rows < 1 || max_new < 1) return set_error(ACTQKV_EINVAL, "n_rows %d or max_new %d < 1", n_rows, max_new);
  if (max_new > n_rows) return set_error(ACTQKV_EINVAL, "max_new %d > n_rows %d", max_new, n_rows);
  if (n_rows > kMaxPagedRows) return set_error(ACTQKV_ESHAPE, "n_rows %d > %d", n_rows, kMaxPagedRows);
  return ACTQKV_OK;
}

static int attention_call(const char* name, const actqkv_shape* shape, int batch, int n_rows, int max_new, const void* q,
                          const int32_t* row_start, const int32_t* n_ctx, const int32_t* pages, int max_pages,
                          const void* k_pages, const void* v_pages, int n_pages, float softcap, int window,
                          const float* slopes, const int32_t* row_first, const int32_t* row_end, void* out, float* lse,
                          const PagedWeights* weights, void* workspace, size_t ws_bytes, void* stream) {
  ACTQKV_TRY(check_table(shape, batch, n_ctx, pages, max_pages, k_pages, v_pages, n_pages));
  ACTQKV_TRY(check_rows(n_rows, max_new));
  // (a launch has less than 2^32 threads: 512 for 64 (row, query head) pairs or, of the account, 128 tokens of a KV head)
  if (int64_t(n_rows) * shape->n_q_heads > 1 << 28)
    return set_error(ACTQKV_ESHAPE, "%d rows of %d query heads > 2^28", n_rows, shape->n_q_heads);
  if (weights != nullptr && int64_t(max_pages) * shape->n_kv_heads > 1 << 22)
    return set_error(ACTQKV_ESHAPE, "weights of %d pages of %d KV heads > 2^22", max_pages, shape->n_kv_heads);
  ACTQKV_REQUIRE_PTR(q);
  ACTQKV_REQUIRE_SMALL(row_start, 4);
  ACTQKV_REQUIRE_PTR(out);
  if (softcap != 0.f && !(softcap >= kLeastCap && softcap <= kLargestCap))
    return set_error(ACTQKV_EINVAL, "softcap must be 0 (none) or between %g and %g", kLeastCap, kLargestCap);
  if (window < 0) return set_error(ACTQKV_EINVAL, "window %d < 0", window);
  ACTQKV_OPTIONAL_SMALL(slopes, 4);
  ACTQKV_OPTIONAL_SMALL(row_first, 4);
  ACTQKV_OPTIONAL_SMALL(row_end, 4);
  ACTQKV_OPTIONAL_SMALL(lse, 4);
  if (weights != nullptr) {
    ACTQKV_REQUIRE_SMALL(lse, 4);
    const float *weights_in = weights->in, *weights_out = weights->out;
    ACTQKV_REQUIRE_PTR(weights_in);
    ACTQKV_REQUIRE_PTR(weights_out);
    if (weights->rows < 1) return set_error(ACTQKV_EINVAL, "weight_rows %d < 1", weights->rows);
    if (weights->stride < int64_t(max_pages) * kBlock)
      return set_error(ACTQKV_EINVAL, "weight_stride %lld < %d pages of %d tokens", (long long)weights->stride, max_pages, kBlock);
    if (weights->stride % 4 != 0) return set_error(ACTQKV_EALIGN, "weight_stride must be a multiple of 4");
  }
  if (workspace == nullptr || !aligned16(workspace))
    return set_error(ACTQKV_EWORKSPACE, "workspace is NULL or not 16-byte aligned");
  const size_t need = paged_workspace_bytes(*shape, batch, n_rows, max_new, max_pages);
  if (ws_bytes < need)
    return set_error(ACTQKV_EWORKSPACE, "workspace has %zu bytes, %s needs %zu", ws_bytes, name, need);
  const float scale = shape->softmax_scale > 0.f ? shape->softmax_scale : 1.f / std::sqrt(float(shape->head_dim));
  PagedAttn p;
  p.t = PagedTable{row_start, n_ctx, pages, batch, n_rows, max_new, max_pages, n_pages, 0};
  p.f = PagedForm{row_first, row_end, slopes, window, scale * kLog2e, softcap > 0.f ? scale / softcap : 0.f, softcap * kLog2e};
  p.n_q_heads = shape->n_q_heads;
  p.n_kv_heads = shape->n_kv_heads;
  p.q = q;
  p.k_pages = k_pages;
  p.v_pages = v_pages;
  p.out = out;
  p.lse = lse;
  return launch_paged_attention(*shape, p, weights, Workspace{workspace, ws_bytes}, static_cast<hipStream_t>(stream));
}

}  // namespace actqkv

using namespace actqkv;

extern "C" {

size_t actqkv_paged_workspace_bytes(const actqkv_shape* shape, int batch, int n_rows, int max_new, int max_pages) {
  if (check_shape(shape) != ACTQKV_OK || check_batch(batch) != ACTQKV_OK) return 0;
  if (check_rows(n_rows, max_new) != ACTQKV_OK) return 0;
  if (max_pages < 1 || max_pages > kMaxPages) {
    set_error(ACTQKV_EINVAL, "paged_workspace_bytes: max_pages %d outside 1..%d", max_pages, kMaxPages);
    return 0;
  }
  return paged_workspace_bytes(*shape, batch, n_rows, max_new, max_pages);
}

int actqkv_paged_append(const actqkv_shape* shape, int batch, int n_rows, int max_new, const void* k_new,
                        const void* v_new, const int32_t* row_start, const int32_t* n_ctx, const int32_t* pages,
                        int max_pages, void* k_pages, void* v_pages, int n_pages, void* stream) {
  ACTQKV_TRY(check_table(shape, batch, n_ctx, pages, max_pages, k_pages, v_pages, n_pages));
  ACTQKV_TRY(check_rows(n_rows, max_new));
  ACTQKV_REQUIRE_PTR(k_new);
  ACTQKV_REQUIRE_PTR(v_new);
  ACTQKV_REQUIRE_SMALL(row_start, 4);
  const PagedTable t{row_start, n_ctx, pages, batch, n_rows, max_new, max_pages, n_pages, 0};
  return launch_paged_append(*shape, t, k_new, v_new, k_pages, v_pages, static_cast<hipStream_t>(stream));
}

int actqkv_paged_attention(const actqkv_shape* shape, int batch, int n_rows, int max_new, const void* q,
                           const int32_t* row_start, const int32_t* n_ctx, const int32_t* pages, int max_pages,
                           const void* k_pages, const void* v_pages, int n_pages, float softcap, int window,
                           const float* slopes, const int32_t* row_first, const int32_t* row_end, void* out, float* lse,
                           void* workspace, size_t ws_bytes, void* stream) {
  return attention_call("paged_attention", shape, batch, n_rows, max_new, q, row_start, n_ctx, pages, max_pages, k_pages,
                        v_pages, n_pages, softcap, window, slopes, row_first, row_end, out, lse, nullptr, workspace,
                        ws_bytes, stream);
}

int actqkv_paged_attention_weights(const actqkv_shape* shape, int batch, int n_rows, int max_new, const void* q,
                                   const int32_t* row_start, const int32_t* n_ctx, const int32_t* pages, int max_pages,
                                   const void* k_pages, const void* v_pages, int n_pages, float softcap, int window,
                                   const float* slopes, const int32_t* row_first, const int32_t* row_end, void* out,
                                   float* lse, int weight_rows, const float* weights_in, float* weights_out,
                                   int64_t weight_stride, void* workspace, size_t ws_bytes, void* stream) {
  const PagedWeights w{weight_rows, weights_in, weights_out, weight_stride};
  return attention_call("paged_attention_weights", shape, batch, n_rows, max_new, q, row_start, n_ctx, pages, max_pages,
                        k_pages, v_pages, n_pages, softcap, window, slopes, row_first, row_end, out, lse, &w, workspace,
                        ws_bytes, stream);
}

int actqkv_paged_evict(const actqkv_shape* shape, int batch, const int32_t* n_ctx, const int32_t* pages, int max_pages,
                       void* k_pages, void* v_pages, int n_pages, const float* weights, int64_t weight_stride,
                       int keep_first, int keep_last, int budget, const int32_t* to_pages, int to_max_pages,
                       float* to_weights, int64_t to_weight_stride, int32_t* kept, int32_t* n_kept, void* stream) {
  ACTQKV_TRY(check_table(shape, batch, n_ctx, pages, max_pages, k_pages, v_pages, n_pages));
  ACTQKV_REQUIRE_SMALL(weights, 4);
  if (weight_stride < int64_t(max_pages) * kBlock)
    return set_error(ACTQKV_EINVAL, "weight_stride %lld < %d pages of %d tokens", (long long)weight_stride, max_pages, kBlock);
  if (to_pages == nullptr || to_pages == pages) {
    if (to_pages != nullptr && to_max_pages != max_pages)
      return set_error(ACTQKV_EINVAL, "in place, but to_max_pages %d is not max_pages %d", to_max_pages, max_pages);
    to_pages = pages;
    to_max_pages = max_pages;
  }
  ACTQKV_REQUIRE_SMALL(to_pages, 4);
  if (to_max_pages < 1) return set_error(ACTQKV_EINVAL, "to_max_pages %d < 1", to_max_pages);
  if (to_max_pages > kMaxPages) return set_error(ACTQKV_ESHAPE, "to_max_pages %d > %d", to_max_pages, kMaxPages);
  if (keep_first < 0 || keep_last < 0 || budget < 1)
    return set_error(ACTQKV_EINVAL, "keep_first %d, keep_last %d negative or budget %d < 1", keep_first, keep_last, budget);
  if (int64_t(keep_first) + keep_last > budget)
    return set_error(ACTQKV_EINVAL, "keep_first %d + keep_last %d > budget %d", keep_first, keep_last, budget);
  if (budget > int64_t(to_max_pages) * kBlock)
    return set_error(ACTQKV_EINVAL, "budget %d > %d pages of %d tokens", budget, to_max_pages, kBlock);
  ACTQKV_OPTIONAL_SMALL(to_weights, 4);
  if (to_weights != nullptr && to_weight_stride < int64_t(to_max_pages) * kBlock)
    return set_error(ACTQKV_EINVAL, "to_weight_stride %lld < %d pages of %d tokens", (long long)to_weight_stride,
                     to_max_pages, kBlock);
  if (to_weights == weights && to_weight_stride != weight_stride)
    return set_error(ACTQKV_EINVAL, "to_weights is weights, but their strides differ");
  ACTQKV_REQUIRE_SMALL(kept, 4);
  ACTQKV_REQUIRE_SMALL(n_kept, 4);
  if (n_kept == n_ctx) return set_error(ACTQKV_EINVAL, "n_kept must not be n_ctx");
  PagedEvict e;
  e.t = PagedTable{nullptr, n_ctx, pages, batch, 0, 0, max_pages, n_pages, 0};
  e.k_pages = k_pages;
  e.v_pages = v_pages;
  e.weights = weights;
  e.stride = weight_stride;
  e.keep_first = keep_first;
  e.keep_last = keep_last;
  e.budget = budget;
  e.to_pages = to_pages;
  e.to_max_pages = to_max_pages;
  e.to_weights = to_weights;
  e.to_stride = to_weight_stride;
  e.kept = kept;
  e.n_kept = n_kept;
  e.n_kv_heads = shape->n_kv_heads;
  return launch_paged_evict(*shape, e, static_cast<hipStream_t>(stream));
}

}  // extern "C"
