// Attention of chunks and prompts over a paged cache in 8 bits, fp32 queries (paged_chunk_f32_body.h has the kernel, paged_chunk_f32.hip its
// design).  Bound by a wavefront's chain of products, softmax and cutting of the probabilities into parts: a tile is 1.6 us where the matrix instructions
// are 0.64.  2 x 2048 rows at 8192 tokens, 8 query and 2 KV heads of 64, 187 to 197 us (over fp32 353 to 366), of 128 458 (774); a prefix of three prompts of
// up to 1500 tokens 24.5 and 6 of merging.  (Two tiles in LDS, a barrier a tile: the same with 64 channels, 3 % slower with 128.)
#include "paged_chunk_f32_body.h"

namespace actqkv {

template <int D, bool kCap, bool kBias>
__global__ __launch_bounds__(kP4Threads, D == 64 ? 2 : 1) void paged8_chunk_f32_kernel(PagedChunkF32 c) {
  chunk_f32_body<D, kCap, kBias, true, false>(c);
}

template <int D>
static void launch_chunk8_f32(const PagedChunkF32& c, hipStream_t stream) {
  const bool cap = c.a.f.cap_in > 0.f, bias = c.a.f.slopes != nullptr;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(unsigned(c.tiles) * c.splits * c.a.n_kv_heads), dim3(kP4Threads), 0, stream, c);
  };
  if (cap && bias) launch(paged8_chunk_f32_kernel<D, true, true>);
  else if (cap) launch(paged8_chunk_f32_kernel<D, true, false>);
  else if (bias) launch(paged8_chunk_f32_kernel<D, false, true>);
  else launch(paged8_chunk_f32_kernel<D, false, false>);
  launch_chunk_f32_merge(D, c, stream);
}
int launch_paged8_chunk_f32(const actqkv_shape& sh, const PagedAttn& p, const Workspace& ws, hipStream_t stream) {
  PagedChunkF32 c;
  c.a = p;
  c.tiles = chunk_f32_tiles(sh, p.t.batch, p.t.n_rows, p.t.max_new);
  c.splits = chunk_f32_splits(sh, p, c.tiles);
  c.part = ws.scratch_f32();
  c.chosen = PagedBits{nullptr, 0};
  if (sh.head_dim == 64) launch_chunk8_f32<64>(c, stream);
  else launch_chunk8_f32<128>(c, stream);
  return hip_status("paged attention (8 bits, chunks, fp32)");
}

}  // namespace actqkv
