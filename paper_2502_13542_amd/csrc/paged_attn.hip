// Attention of new tokens over a paged cache: a workgroup per (row, query head), a key per thread, one pass over the
// pages with the running maximum and sum; then the attention weight, a key per thread.
#include <cmath>

#include "paged.h"

namespace actqkv {

constexpr int kPsThreads = kBlock;

template <typename T, int D, bool kCap, bool kBias>
__global__ __launch_bounds__(kPsThreads) void paged_attention_kernel(PagedAttn p) {
  __shared__ float ql[D], pl[kBlock], red[32];
  const int row = blockIdx.x, head = blockIdx.y, tid = threadIdx.x;
  const int hk = head / (p.n_q_heads / p.n_kv_heads);
  int s = 0;
  while (s + 1 < p.t.batch && p.t.row_start[s + 1] <= row) ++s;
  const PagedSeq seq = paged_seq(p.t, s);
  if (row < seq.row0 || row >= seq.row0 + seq.m) return;
  const int pos = seq.n - seq.m + (row - seq.row0);
  const PagedSpan v = paged_span(p.f, row, pos, seq.n);
  const float slope = kBias ? p.f.slopes[head] * kLog2e : 0.f;
  const T* qp = static_cast<const T*>(p.q) + (size_t(row) * p.n_q_heads + head) * D;
  if (tid < D) ql[tid] = to_f32(qp[tid]);
  __syncthreads();
  float m_run = -INFINITY, l_run = 0.f, o = 0.f;
  const int t_end = v.hi > v.lo ? (v.hi + kBlock - 1) / kBlock : 0;
  for (int t = v.lo / kBlock; t < t_end; ++t) {
    const int page = paged_page(p.t, s, t);
    if (page < 0) continue;
    const size_t tile = (size_t(page) * p.n_kv_heads + hk) * (kBlock * D);
    const int j = t * kBlock + tid;
    float sc = -INFINITY;
    if (j >= v.lo && j < v.hi) {
      const T* kp = static_cast<const T*>(p.k_pages) + tile + size_t(tid) * D;
      float dot = 0.f;
      for (int d = 0; d < D; ++d) dot = fmaf(to_f32(kp[d]), ql[d], dot);
      sc = paged_score<kCap, kBias>(p.f, dot, slope, abs(pos - j));
    }
    const float m_new = fmaxf(m_run, block_max(sc, red));
    const float m_safe = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = exp2f(m_run - m_safe), pv = exp2f(sc - m_safe);
    m_run = m_new;
    pl[tid] = pv;
    l_run = l_run * alpha + block_sum(pv, red);
    if (tid < D) {
      const T* vp = static_cast<const T*>(p.v_pages) + tile + size_t(tid) * kBlock;
      o *= alpha;
      for (int k = max(v.lo - t * kBlock, 0); k < min(v.hi - t * kBlock, kBlock); ++k) o = fmaf(pl[k], to_f32(vp[k]), o);
    }
    __syncthreads();
  }
  if (tid < D) store_elem(static_cast<T*>(p.out) + (size_t(row) * p.n_q_heads + head) * D + tid, l_run > 0.f ? o / l_run : 0.f);
  if (tid == 0 && p.lse != nullptr) p.lse[size_t(row) * p.n_q_heads + head] = (m_run + log2f(l_run)) * kLn2;
}

size_t paged_workspace_bytes(const actqkv_shape& sh, int batch, int n_rows, int max_new, int max_pages) {
  return kCounterBytes + align_up(std::max({paged_step_scratch_most(sh, batch, max_new, max_pages),
                                            paged_chunk_scratch_most(sh, batch, n_rows, max_new, max_pages),
                                            paged_votes_scratch_most(sh)}), 256);
}

template <int D>
static void launch_form(const PagedAttn& p, hipStream_t stream) {
  const bool cap = p.f.cap_in > 0.f, bias = p.f.slopes != nullptr;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(p.t.n_rows, p.n_q_heads), dim3(kPsThreads), 0, stream, p);
  };
  if (cap && bias) launch(paged_attention_kernel<float, D, true, true>);
  else if (cap) launch(paged_attention_kernel<float, D, true, false>);
  else if (bias) launch(paged_attention_kernel<float, D, false, true>);
  else launch(paged_attention_kernel<float, D, false, false>);
}
int launch_paged_attention(const actqkv_shape& sh, const PagedAttn& p, const PagedWeights* weights, const Workspace& ws,
                           hipStream_t stream) {
  if (paged_step_supported(sh, p.t.max_new)) return launch_paged_step(sh, p, weights, ws, stream);
  int rc;
  if (paged_chunk_supported(sh)) {
    rc = launch_paged_chunk(sh, p, ws, stream);
  } else {
    if (sh.head_dim == 64) launch_form<64>(p, stream);
    else launch_form<128>(p, stream);
    rc = hip_status("paged attention");
  }
  if (rc != ACTQKV_OK || weights == nullptr) return rc;
  return launch_paged_votes(sh, p, *weights, ws, stream);
}

}  // namespace actqkv
