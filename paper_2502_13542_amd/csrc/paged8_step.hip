// Attention over a paged cache in 8 bits of sequences that bring few rows (paged_step_body.h has the kernel, paged8_shape.h the operands
// of an item, a page of 128 keys: as many bytes on their way as of 64 keys in 16 bits).  Bound by HBM: 16 sequences at up to 32K tokens, 32 query and
// 8 KV heads of 128, 707 MB, 148 us = 4.8 TB/s (pages in 16 bits: twice the bytes, 265 to 272); 1 at 32K 19 us, 48 at up to 8K 116; one of 700 tokens,
// small fp32 model, 7.  (256 threads a workgroup, two of them resident: 155, 1 at 32K 24; loads that pass the caches by: 172, since two of them share a line.)
#include "paged8_shape.h"
#include "paged_step_body.h"

namespace actqkv {

// (At least two wavefronts a SIMD: two workgroups of four on a compute unit.  Left to itself the compiler takes up to 290 registers for fp32 and 128
// channels, and 258 for bf16 under a cap with slopes; so 3 to 8 of fp32 with 128 channels are in scratch, of workgroups of eight as well.)
template <typename T, int D, int W, bool kCap, bool kBias>
__global__ __launch_bounds__(64 * W, 2) void paged8_step_kernel(PagedStep st) {
  step_body<Step8Shape<T, D>, T, D, kCap, kBias, false, W>(st);
}
template <typename T, int D, int W>
static void launch_step8_by(const PagedStep& st, hipStream_t stream) {
  const bool cap = st.a.f.cap_in > 0.f, bias = st.a.f.slopes != nullptr;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(st.n_wg, st.a.n_kv_heads, st.a.t.batch), dim3(64 * W), 0, stream, st);
  };
  if (cap && bias) launch(paged8_step_kernel<T, D, W, true, true>);
  else if (cap) launch(paged8_step_kernel<T, D, W, true, false>);
  else if (bias) launch(paged8_step_kernel<T, D, W, false, true>);
  else launch(paged8_step_kernel<T, D, W, false, false>);
}
// Many short sequences by workgroups of four wavefronts, two of them on a compute unit: more workgroups than there are compute units, of a page for each
// wavefront, or half as many again of up to 16.  us of eight | four, 32 query and 8 KV heads of 128: 300 sequences at up to 128 tokens 47 | 30, 64 at 700
// 20.6 | 17.4, at 2K 40 | 34, at 8K (32 a workgroup) 150 | 150, 33 at 1K 17.9 | 20.0; 28 and 4 heads, 42 at 724 (3) 17.5 | 14.4, 80 at 724 (6) 18.8 | 20.8, 80
// at 3K 42 | 51; fp32, 8 and 2 heads of 64, 200 at 1K 15.3 | 13.7, of 128 100 at 1K 21.9 | 18.0,
// 32 and 8 heads 300 at up to 128 62 | 36, 64 at 2K 50 | 43, 33 at 700 18.0 | 19.0; under a cap with slopes, bf16, 300 at up to 128 60 | 34, 64 at 2K 49 | 40; fewer workgroups: 32 and 8 heads, 32 at 700 10.9 | 11.9.
template <typename T, int D>
static void launch_step8(const PagedStep& st, hipStream_t stream) {
  const int64_t wgs = int64_t(st.a.t.batch) * st.a.n_kv_heads * st.n_wg, pages = (st.a.t.max_pages + st.n_wg - 1) / st.n_wg;
  if ((wgs > kChipCus && pages <= 4) || (2 * wgs >= 3 * kChipCus && pages <= 16)) launch_step8_by<T, D, 4>(st, stream);
  else launch_step8_by<T, D, 8>(st, stream);
}
size_t paged8_step_scratch_most(const actqkv_shape& sh, int batch) { return step_part_most(sh, int64_t(batch) * sh.n_kv_heads); }
int launch_paged8_step(const actqkv_shape& sh, const PagedAttn& p, const Workspace& ws, hipStream_t stream) {
  PagedStep st = {};
  st.a = p;
  st.n_wg = step_workgroups(int64_t(p.t.batch) * sh.n_kv_heads, p.t.max_pages, step_least(kBlock, sh.head_dim, 1), 4);
  st.part = reinterpret_cast<uint32_t*>(ws.scratch_f32());
  st.counters = ws.counters();
  if (sh.dtype == ACTQKV_F32) {
    if (sh.head_dim == 64) launch_step8<float, 64>(st, stream);
    else launch_step8<float, 128>(st, stream);
  } else {
    if (sh.head_dim == 64) launch_step8<uint16_t, 64>(st, stream);
    else launch_step8<uint16_t, 128>(st, stream);
  }
  return hip_status("paged attention (8 bits, few rows)");
}

}  // namespace actqkv
