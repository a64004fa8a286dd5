// Attention of chunks and prompts over a paged cache in fp32: products on the 16-bit matrix cores, a value as three bf16 parts and
// a product as six of theirs, which keep all of its bits (attn_prefill_f32.hip has the arithmetic and what it is measured to be worth;
// the fp32 matrix instruction does a sixteenth of the 16-bit one's operations).
//
// A workgroup of 4 wavefronts owns 128 query rows that share a KV head (numbered position by position, the G heads side by
// side), a wavefront 32 of them.  A tile is 4096 / D keys of a page, 16 KB of keys and 16 KB of values: every wavefront brings a quarter
// of each into registers while the tile before is worked on, and cuts it into parts in LDS (48 KB, one tile) between two barriers.
// With 64 channels two workgroups share a compute unit; with 128 one has all of its registers (two, with 73 in scratch, were 10 % slower).
// 2 x 2048 rows at 8192 tokens, 8 query and 2 KV heads of 64: 353 to 366 us (164 to 170 TFLOP/s), of 128: 774 (155); bound by the vector work of cutting
// and softmax and by operand reads beside the products.  (Two tiles in LDS, cut between the products of the one before: 64 channels
// 422, 128 810; three sums of the scores in turn, 128 channels: 803.)  Keys that no row of the workgroup sees enter as zeros, whatever
// their slots hold.  Where the query tiles do not fill the chip the tiles are cut into pieces that a second launch merges.
#include "paged_chunk_f32_body.h"

namespace actqkv {

template <int D, bool kCap, bool kBias>
__global__ __launch_bounds__(kP4Threads, D == 64 ? 2 : 1) void paged_chunk_f32_kernel(PagedChunkF32 c) {
  chunk_f32_body<D, kCap, kBias, false, false>(c);
}

size_t paged_chunk_f32_scratch_most(const actqkv_shape& sh, int batch, int n_rows, int max_new, int max_pages, bool byte) {
  if (sh.dtype != ACTQKV_F32) return 0;
  const int64_t pieces = std::min<int64_t>(kP4MaxSplits, int64_t(max_pages) * (kBlock / (4096 / sh.head_dim))) * sh.n_kv_heads *
                         chunk_f32_tiles(sh, batch, n_rows, max_new);
  return size_t(std::min<int64_t>(byte ? kP4SlotsByte : kP4Slots, pieces)) * (sh.head_dim == 64 ? ChunkPieceF32<64>::bytes() : ChunkPieceF32<128>::bytes());
}

void launch_chunk_f32_merge(int d, const PagedChunkF32& c, hipStream_t stream) {
  const PagedMerge merge{c.a, c.tiles, c.splits, c.part};
  if (c.splits == 1) return;
  if (d == 64) launch_paged_merge<float, 64, kP4Waves, 2, 1>(merge, stream);
  else launch_paged_merge<float, 128, kP4Waves, 4, 1>(merge, stream);
}

template <int D>
static void launch_chunk_f32(const PagedChunkF32& c, hipStream_t stream) {
  const bool cap = c.a.f.cap_in > 0.f, bias = c.a.f.slopes != nullptr;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(unsigned(c.tiles) * c.splits * c.a.n_kv_heads), dim3(kP4Threads), 0, stream, c);
  };
  if (cap && bias) launch(paged_chunk_f32_kernel<D, true, true>);
  else if (cap) launch(paged_chunk_f32_kernel<D, true, false>);
  else if (bias) launch(paged_chunk_f32_kernel<D, false, true>);
  else launch(paged_chunk_f32_kernel<D, false, false>);
  launch_chunk_f32_merge(D, c, stream);
}
void paged_chunk_f32_cut(const actqkv_shape& sh, const PagedAttn& p, int32_t* cut) {
  cut[0] = kP4Rows;
  cut[1] = 1;
  cut[2] = chunk_f32_splits(sh, p, chunk_f32_tiles(sh, p.t.batch, p.t.n_rows, p.t.max_new));
}
int launch_paged_chunk_f32(const actqkv_shape& sh, const PagedAttn& p, const Workspace& ws, hipStream_t stream) {
  PagedChunkF32 c;
  c.a = p;
  c.tiles = chunk_f32_tiles(sh, p.t.batch, p.t.n_rows, p.t.max_new);
  c.splits = chunk_f32_splits(sh, p, c.tiles);
  c.part = ws.scratch_f32();
  c.chosen = PagedBits{nullptr, 0};
  if (sh.head_dim == 64) launch_chunk_f32<64>(c, stream);
  else launch_chunk_f32<128>(c, stream);
  return hip_status("paged attention (chunks, fp32)");
}

}  // namespace actqkv
