// Attention of rows that look at selected pages each (paged_step_body.h has the kernel): a (row, KV head) of its own per group of
// workgroups, its items the halves of the pages in the row's list.
#include "paged_step_body.h"

namespace actqkv {

template <typename T, int D, bool kCap, bool kBias>
__global__ __launch_bounds__(kStThreads) void paged_selected_kernel(PagedStep st) {
  step_body<StepShape<T, D>, T, D, kCap, kBias, true>(st);
}
template <typename T, int D>
static void launch_selected(const PagedStep& st, hipStream_t stream) {
  const bool cap = st.a.f.cap_in > 0.f, bias = st.a.f.slopes != nullptr;
  const unsigned n = unsigned(st.a.t.n_rows) * st.a.n_kv_heads * st.n_wg;
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(n), dim3(kStThreads), 0, stream, st); };
  if (cap && bias) launch(paged_selected_kernel<T, D, true, true>);
  else if (cap) launch(paged_selected_kernel<T, D, true, false>);
  else if (bias) launch(paged_selected_kernel<T, D, false, true>);
  else launch(paged_selected_kernel<T, D, false, false>);
}
size_t paged_selected_scratch_most(const actqkv_shape& sh, int n_rows) {
  return step_part_most(sh, int64_t(n_rows) * sh.n_kv_heads);
}
int launch_paged_selected(const actqkv_shape& sh, const PagedAttn& p, const int32_t* idx, const int32_t* n_sel, int k_sel,
                          const Workspace& ws, hipStream_t stream) {
  const bool f32 = sh.dtype == ACTQKV_F32;
  const int keys = f32 ? 4096 / sh.head_dim : 64;
  PagedStep st = {};
  st.a = p;
  st.n_wg = step_workgroups(int64_t(p.t.n_rows) * sh.n_kv_heads, int64_t(std::min(k_sel, p.t.max_pages)) * (kBlock / keys),
                            step_least(keys, sh.head_dim, f32 ? 4 : 2));
  st.part = reinterpret_cast<uint32_t*>(ws.scratch_f32());
  st.counters = ws.counters();
  st.idx = idx;
  st.n_sel = n_sel;
  st.k_sel = k_sel;
  if (f32) {
    if (sh.head_dim == 64) launch_selected<float, 64>(st, stream);
    else launch_selected<float, 128>(st, stream);
  } else {
    if (sh.head_dim == 64) launch_selected<uint16_t, 64>(st, stream);
    else launch_selected<uint16_t, 128>(st, stream);
  }
  return hip_status("paged attention (selected pages)");
}

}  // namespace actqkv
