// Attention of chunks and prompts over a paged cache in 8 bits, bf16 queries (paged_chunk_body.h has the kernel, paged_chunk.hip its design).
// Bound as over 16 bits: 2 x 2048 rows at 16K tokens, 32 query and 8 KV heads of 128, 905 to 980 us between cards (1.05 to 1.14 PFLOP/s; 8192^3 as a library
// product 1.20 to 1.23), mixed rows under a cap and a window, 28 and 4 heads, 257 to 266 (260 over 16 bits): the codes' conversion, 32 instructions a wavefront
// and page, is hidden.  The cut goes by figures of its own (chunk_cut).  With 256 rows, 128 channels and slopes 10 registers are in scratch.
#include "paged_chunk_body.h"

namespace actqkv {

template <int D, int KS, bool kCap, bool kBias>
__global__ __launch_bounds__(kPcThreads) void paged8_chunk_kernel(PagedChunk c) {
  chunk_body<D, KS, kCap, kBias, true, false>(c);
}

template <int D, int KS>
static void launch_chunk8(const PagedChunk& c, hipStream_t stream) {
  const bool cap = c.a.f.cap_in > 0.f, bias = c.a.f.slopes != nullptr;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(unsigned(c.tiles) * c.splits * c.a.n_kv_heads), dim3(kPcThreads), 0, stream, c);
  };
  if (cap && bias) launch(paged8_chunk_kernel<D, KS, true, true>);
  else if (cap) launch(paged8_chunk_kernel<D, KS, true, false>);
  else if (bias) launch(paged8_chunk_kernel<D, KS, false, true>);
  else launch(paged8_chunk_kernel<D, KS, false, false>);
  launch_chunk_merge(D, KS, c, stream);
}
template <int D>
static void launch_chunk8_ks(int ks, const PagedChunk& c, hipStream_t stream) {
  if (ks == 1) launch_chunk8<D, 1>(c, stream);
  else if (ks == 2) launch_chunk8<D, 2>(c, stream);
  else launch_chunk8<D, 4>(c, stream);
}
int launch_paged8_chunk(const actqkv_shape& sh, const PagedAttn& p, const Workspace& ws, hipStream_t stream) {
  const ChunkCut cut = chunk_cut(sh, p);
  PagedChunk c;
  c.a = p;
  c.tiles = cut.tiles;
  c.splits = cut.splits;
  c.part = ws.scratch_f32();
  c.chosen = PagedBits{nullptr, 0};
  if (sh.head_dim == 64) launch_chunk8_ks<64>(cut.ks, c, stream);
  else launch_chunk8_ks<128>(cut.ks, c, stream);
  return hip_status("paged attention (8 bits, chunks)");
}

}  // namespace actqkv
