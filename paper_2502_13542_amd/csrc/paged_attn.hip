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

template <typename T, int D, bool kCap, bool kBias>
__global__ __launch_bounds__(kPsThreads) void paged_weights_kernel(PagedAttn p, PagedWeights w) {
  __shared__ float ql[D];
  const int t = blockIdx.x, hk = blockIdx.y, s = blockIdx.z, tid = threadIdx.x;
  const int group = p.n_q_heads / p.n_kv_heads, j = t * kBlock + tid;
  const PagedSeq seq = paged_seq(p.t, s);
  const int page = paged_page(p.t, s, t);
  float sum = 0.f;
  if (page >= 0) {
    const T* kp = static_cast<const T*>(p.k_pages) + (size_t(page) * p.n_kv_heads + hk) * (kBlock * D) + size_t(tid) * D;
    for (int i = max(seq.m - w.rows, 0); i < seq.m; ++i) {
      const int row = seq.row0 + i, pos = seq.n - seq.m + i;
      const PagedSpan v = paged_span(p.f, row, pos, seq.n);
      for (int g = 0; g < group; ++g) {
        const int head = hk * group + g;
        const T* qp = static_cast<const T*>(p.q) + (size_t(row) * p.n_q_heads + head) * D;
        __syncthreads();
        if (tid < D) ql[tid] = to_f32(qp[tid]);
        __syncthreads();
        const float lse = p.lse[size_t(row) * p.n_q_heads + head];
        if (j >= v.lo && j < v.hi && lse > -INFINITY) {
          float dot = 0.f;
          for (int d = 0; d < D; ++d) dot = fmaf(to_f32(kp[d]), ql[d], dot);
          const float slope = kBias ? p.f.slopes[head] * kLog2e : 0.f;
          sum += exp2f(paged_score<kCap, kBias>(p.f, dot, slope, abs(pos - j)) - lse * kLog2e);
        }
      }
    }
  }
  const size_t at = (size_t(s) * p.n_kv_heads + hk) * w.stride + j;
  w.out[at] = w.in[at] + sum;
}

size_t paged_workspace_bytes(const actqkv_shape& sh, int batch, int n_rows, int max_new, int max_pages) {
  return kCounterBytes + align_up(std::max(paged_step_scratch_most(sh, batch, max_new, max_pages),
                                           paged_chunk_scratch_most(sh, batch, n_rows, max_new, max_pages)), 256);
}

template <typename T, int D, bool kCap, bool kBias>
static void launch_both(const PagedAttn& p, const PagedWeights* w, bool attend, hipStream_t stream) {
  if (attend) hipLaunchKernelGGL((paged_attention_kernel<T, D, kCap, kBias>), dim3(p.t.n_rows, p.n_q_heads), dim3(kPsThreads), 0, stream, p);
  if (w != nullptr)
    hipLaunchKernelGGL((paged_weights_kernel<T, D, kCap, kBias>), dim3(p.t.max_pages, p.n_kv_heads, p.t.batch),
                       dim3(kPsThreads), 0, stream, p, *w);
}
template <typename T, int D>
static void launch_form(const PagedAttn& p, const PagedWeights* w, bool attend, hipStream_t stream) {
  const bool cap = p.f.cap_in > 0.f, bias = p.f.slopes != nullptr;
  if (cap && bias) launch_both<T, D, true, true>(p, w, attend, stream);
  else if (cap) launch_both<T, D, true, false>(p, w, attend, stream);
  else if (bias) launch_both<T, D, false, true>(p, w, attend, stream);
  else launch_both<T, D, false, false>(p, w, attend, stream);
}
int launch_paged_attention(const actqkv_shape& sh, const PagedAttn& p, const PagedWeights* weights, const Workspace& ws,
                           hipStream_t stream) {
  if (paged_step_supported(sh, p.t.max_new)) return launch_paged_step(sh, p, weights, ws, stream);
  const bool attend = !paged_chunk_supported(sh);
  if (!attend)
    if (int rc = launch_paged_chunk(sh, p, ws, stream)) return rc;
  if (sh.dtype == ACTQKV_F32) {
    if (sh.head_dim == 64) launch_form<float, 64>(p, weights, attend, stream);
    else launch_form<float, 128>(p, weights, attend, stream);
  } else {
    if (sh.head_dim == 64) launch_form<uint16_t, 64>(p, weights, attend, stream);
    else launch_form<uint16_t, 128>(p, weights, attend, stream);
  }
  return hip_status("paged attention");
}

}  // namespace actqkv
