// Attention of chunks of fp32 rows that look at selected pages each (paged_chunk_f32_body.h has the kernel, paged_chunk_f32.hip its design).
#include "paged_chunk_f32_body.h"

namespace actqkv {

template <int D, bool kCap, bool kBias>
__global__ __launch_bounds__(kP4Threads, D == 64 ? 2 : 1) void paged_chosen_chunk_f32_kernel(PagedChunkF32 c) {
  chunk_f32_body<D, kCap, kBias, false, true>(c);
}

template <int D>
static void launch_chosen_f32(const PagedChunkF32& c, hipStream_t stream) {
  const bool cap = c.a.f.cap_in > 0.f, bias = c.a.f.slopes != nullptr;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(unsigned(c.tiles) * c.splits * c.a.n_kv_heads), dim3(kP4Threads), 0, stream, c);
  };
  if (cap && bias) launch(paged_chosen_chunk_f32_kernel<D, true, true>);
  else if (cap) launch(paged_chosen_chunk_f32_kernel<D, true, false>);
  else if (bias) launch(paged_chosen_chunk_f32_kernel<D, false, true>);
  else launch(paged_chosen_chunk_f32_kernel<D, false, false>);
  launch_chunk_f32_merge(D, c, stream);
}
double paged_chosen_chunk_f32_us(const actqkv_shape& sh, const PagedAttn& p) {
  double us;
  chunk_f32_splits(sh, p, chunk_f32_tiles(sh, p.t.batch, p.t.n_rows, p.t.max_new), &us);
  return us;
}
int launch_paged_chosen_chunk_f32(const actqkv_shape& sh, const PagedAttn& p, const PagedBits& bits, const Workspace& ws, hipStream_t stream) {
  PagedChunkF32 c;
  c.a = p;
  c.tiles = chunk_f32_tiles(sh, p.t.batch, p.t.n_rows, p.t.max_new);
  c.splits = chunk_f32_splits(sh, p, c.tiles);
  c.part = ws.scratch_f32();
  c.chosen = bits;
  if (sh.head_dim == 64) launch_chosen_f32<64>(c, stream);
  else launch_chosen_f32<128>(c, stream);
  return hip_status("paged attention (selected pages, chunks, fp32)");
}

}  // namespace actqkv
