// Attention over a paged cache of sequences that bring few rows: at most 16 (row, query head) pairs per KV head (a decode step,
// a few drafted tokens).  HBM-bound: every key and value byte is read once, by one wavefront.
//
// A wavefront owns work items of up to 64 keys of one (sequence, KV head) whose keys and values are requested together, straight
// into MFMA operands (decode_shape.h); the (row, head) pairs are the columns of its 16-wide products, each with its own span of
// visible keys.  The page of an item is looked up for 64 items at a time, one per lane, so that no item waits for its table
// entry.  The items of a (sequence, KV head) go round the wavefronts of up to n_wg workgroups (as many as it has work for);
// the wavefronts of a workgroup merge (max, sum, O) in LDS, the workgroups through the workspace, in the one that finishes last.
// 16 sequences at up to 32K tokens, 32 query and 8 KV heads of 128, bf16: 265 us = 5.3 TB/s; 8 at up to 16K with the account of weights 100 us,
// 7 of them the second kernel; one of 700 tokens, small fp32 model, 7.7 to 8.8, a chain of round trips.
#include "paged_step_body.h"

namespace actqkv {

template <typename T, int D, bool kCap, bool kBias>
__global__ __launch_bounds__(kStThreads) void paged_step_kernel(PagedStep st) {
  step_body<StepShape<T, D>, T, D, kCap, kBias, false>(st);
}

// The account of the attention weight from the scores that the step kernel kept: four keys a thread.
constexpr int kSwThreads = 256, kSwKeys = 4 * kSwThreads;
__global__ __launch_bounds__(kSwThreads) void paged_step_weights_kernel(PagedStep st, PagedWeights w) {
  const PagedAttn& p = st.a;
  const int hk = blockIdx.y, s = blockIdx.z, group = p.n_q_heads / p.n_kv_heads;
  const int pair = s * p.n_kv_heads + hk, j = blockIdx.x * kSwKeys + threadIdx.x * 4;
  const int keys = p.t.max_pages * kBlock;
  if (j >= keys) return;
  const PagedSeq seq = paged_seq(p.t, s);
  const bool live = j < seq.n && paged_page(p.t, s, j / kBlock) >= 0;
  const size_t at = size_t(pair) * w.stride + j;
  if (!live && w.in == w.out) return;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  const float* scores = st.scores + size_t(pair) * (p.t.max_new * group) * size_t(keys) + j;
  if (live) {
    for (int i = max(seq.m - w.rows, 0); i < seq.m; ++i) {
      const int row = seq.row0 + i;
      const PagedSpan v = paged_span(p.f, row, seq.n - seq.m + i, seq.n);
      if (v.hi <= v.lo || v.hi <= j || v.lo > j + 3) continue;
      for (int g = 0; g < group; ++g) {
        const float lse = p.lse[size_t(row) * p.n_q_heads + hk * group + g] * kLog2e;
        const f32x4 x = *reinterpret_cast<const f32x4*>(scores + size_t(i * group + g) * keys);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += j + e >= v.lo && j + e < v.hi ? __builtin_amdgcn_exp2f(x[e] - lse) : 0.f;
      }
    }
  }
  *reinterpret_cast<f32x4*>(w.out + at) = *reinterpret_cast<const f32x4*>(w.in + at) + sum;
}

// ---- host side
bool paged_step_supported(const actqkv_shape& sh, int max_new) { return int64_t(max_new) * (sh.n_q_heads / sh.n_kv_heads) <= 16; }

static int step_keys(const actqkv_shape& sh) { return sh.dtype == ACTQKV_F32 ? 4096 / sh.head_dim : 64; }

static int step_workgroups(const actqkv_shape& sh, int batch, int max_pages) {
  return step_workgroups(int64_t(batch) * sh.n_kv_heads, int64_t(max_pages) * (kBlock / step_keys(sh)),
                         step_least(step_keys(sh), sh.head_dim, sh.dtype == ACTQKV_F32 ? 4 : 2));
}
static size_t step_part_bytes(const actqkv_shape& sh, int batch, int max_pages) {
  const int n_wg = step_workgroups(sh, batch, max_pages);
  return n_wg == 1 ? 0 : size_t(batch) * sh.n_kv_heads * n_wg * 16 * (sh.head_dim + 2) * sizeof(float);
}
// Enough for every step call of at most so many sequences, rows of one and pages: the partial results only grow with the pages,
// and by the number of sequences are at most those of kStepWgs + pairs workgroups.
size_t paged_step_scratch_most(const actqkv_shape& sh, int batch, int max_new, int max_pages) {
  const int group = sh.n_q_heads / sh.n_kv_heads;
  const size_t cols = size_t(std::min(max_new, 16 / group)) * group;
  return step_part_most(sh, int64_t(batch) * sh.n_kv_heads) + size_t(batch) * sh.n_kv_heads * cols * max_pages * kBlock * sizeof(float);
}

template <typename T, int D>
static void launch_step(const PagedStep& st, hipStream_t stream) {
  const bool cap = st.a.f.cap_in > 0.f, bias = st.a.f.slopes != nullptr;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(st.n_wg, st.a.n_kv_heads, st.a.t.batch), dim3(kStThreads), 0, stream, st);
  };
  if (cap && bias) launch(paged_step_kernel<T, D, true, true>);
  else if (cap) launch(paged_step_kernel<T, D, true, false>);
  else if (bias) launch(paged_step_kernel<T, D, false, true>);
  else launch(paged_step_kernel<T, D, false, false>);
}

int launch_paged_step(const actqkv_shape& sh, const PagedAttn& p, const PagedWeights* weights, const Workspace& ws,
                      hipStream_t stream) {
  PagedStep st;
  st.a = p;
  st.n_wg = step_workgroups(sh, p.t.batch, p.t.max_pages);
  st.part = reinterpret_cast<uint32_t*>(ws.scratch_f32());
  st.counters = ws.counters();
  st.scores = nullptr;
  st.weight_rows = 0;
  st.idx = st.n_sel = nullptr;
  st.k_sel = 0;
  if (weights != nullptr) {
    st.scores = ws.scratch_f32() + align_up(step_part_bytes(sh, p.t.batch, p.t.max_pages), 256) / sizeof(float);
    st.weight_rows = weights->rows;
  }
  if (sh.dtype == ACTQKV_F32) {
    if (sh.head_dim == 64) launch_step<float, 64>(st, stream);
    else launch_step<float, 128>(st, stream);
  } else {
    if (sh.head_dim == 64) launch_step<uint16_t, 64>(st, stream);
    else launch_step<uint16_t, 128>(st, stream);
  }
  if (weights != nullptr) {
    const dim3 grid((p.t.max_pages * kBlock + kSwKeys - 1) / kSwKeys, p.n_kv_heads, p.t.batch);
    hipLaunchKernelGGL(paged_step_weights_kernel, grid, dim3(kSwThreads), 0, stream, st, *weights);
  }
  return hip_status("paged attention (few rows)");
}

}  // namespace actqkv
