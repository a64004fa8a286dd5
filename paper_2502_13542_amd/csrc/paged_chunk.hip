// Attention of chunks and prompts over a paged cache on the matrix cores (bf16 storage, fp32 sums).
//
// Work split.  The query rows of a (sequence, KV head) are numbered position by position, the G heads of the KV head side by
// side; a workgroup of 8 wavefronts takes 256 / KS of them, 32 for KS wavefronts (KS = 1, 2 or 4), which share the keys of every
// page and merge in LDS at the end.  A workgroup finds its sequence by a scan over row_start.  Where that leaves compute units
// idle the pages are cut into pieces, a workgroup each, merged by a second launch (chunk_cut).  Workgroups of one KV head
// sit on few XCDs (blockIdx % Hk), so that the pages they share stay in those L2s.
//
// Data flow per page.  Keys [128][D] and values [D][128] go from HBM straight into LDS (double buffered, 16-byte chunks
// XOR-swizzled with the row, so that operand reads of 16 rows hit all banks).  S^T = K Q^T with v_mfma_f32_32x32x16_bf16 leaves a
// lane with scores of ONE row; the keys enter in an order (bits 2 and 3 of their number exchanged) that makes 8 registers
// of it the B operand of O^T += V^T P^T.  The softmax runs in one pass with a running maximum that follows lazily (it moves when a
// page exceeds it by 2^8), its sum in fp32 before the probabilities are rounded to bf16: the logarithm of that sum is an
// output, and from rounded terms it would have 10 bits.  The rounding of the probabilities costs the output as much as its own
// (1.66e-3 of it each, 2.3e-3 together); keeping what it leaves as a second term costs half as many products again.
//
// Bound by power with whole pages: 2 x 2048 rows at 16K tokens, 32 query and 8 KV heads of 128, 906 to 954 us (1.08 to 1.14 PFLOP/s, the
// matrix pipe busy in 61 % of the cycles at 1.7 GHz; an 8192^3 library product 1.25 to 1.33), under a cap by vector instructions (21 % more; with 256 rows and 128 channels 6 registers are in scratch then, 7 with slopes too).
//
// Every row sees a span of positions.  A page that all rows of a wavefront see whole takes the path without a mask, one that
// none sees is skipped, and the walk is over the union of the spans: a window or documents cost what they cover.
#include "paged_chunk_body.h"

namespace actqkv {

template <int D, int KS, bool kCap, bool kBias>
__global__ __launch_bounds__(kPcThreads) void paged_chunk_kernel(PagedChunk c) {
  chunk_body<D, KS, kCap, kBias, false, false>(c);
}

size_t paged_chunk_scratch_most(const actqkv_shape& sh, int batch, int n_rows, int max_new, int max_pages, bool byte) {
  if (sh.dtype != ACTQKV_BF16) return 0;
  size_t most = 0;
  for (int ks = 1; ks <= 4; ks *= 2)
    most = std::max(most, size_t(std::min(kPcMaxSplits, max_pages)) * sh.n_kv_heads * chunk_tiles(sh, batch, n_rows, max_new, ks) *
                              chunk_piece_bytes(sh, ks));
  return std::min(most, (byte ? kPcMostPiecesByte : kPcMostPieces) * chunk_piece_bytes(sh, 1));
}

template <int D, int KS>
static void launch_merge(const PagedChunk& c, hipStream_t stream) {
  constexpr int kDb = D / 32;
  launch_paged_merge<uint16_t, D, kPcWaves / KS, (kDb > KS ? kDb / KS : 1), (kDb < KS ? kDb : KS)>(
      PagedMerge{c.a, c.tiles, c.splits, c.part}, stream);
}
void launch_chunk_merge(int d, int ks, const PagedChunk& c, hipStream_t stream) {
  if (c.splits == 1) return;
  if (d == 64) {
    if (ks == 1) launch_merge<64, 1>(c, stream);
    else if (ks == 2) launch_merge<64, 2>(c, stream);
    else launch_merge<64, 4>(c, stream);
  } else {
    if (ks == 1) launch_merge<128, 1>(c, stream);
    else if (ks == 2) launch_merge<128, 2>(c, stream);
    else launch_merge<128, 4>(c, stream);
  }
}

template <int D, int KS>
static void launch_chunk(const PagedChunk& c, hipStream_t stream) {
  const bool cap = c.a.f.cap_in > 0.f, bias = c.a.f.slopes != nullptr;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(unsigned(c.tiles) * c.splits * c.a.n_kv_heads), dim3(kPcThreads), 0, stream, c);
  };
  if (cap && bias) launch(paged_chunk_kernel<D, KS, true, true>);
  else if (cap) launch(paged_chunk_kernel<D, KS, true, false>);
  else if (bias) launch(paged_chunk_kernel<D, KS, false, true>);
  else launch(paged_chunk_kernel<D, KS, false, false>);
  launch_chunk_merge(D, KS, c, stream);
}
template <int D>
static void launch_chunk_ks(int ks, const PagedChunk& c, hipStream_t stream) {
  if (ks == 1) launch_chunk<D, 1>(c, stream);
  else if (ks == 2) launch_chunk<D, 2>(c, stream);
  else launch_chunk<D, 4>(c, stream);
}
void paged_chunk_cut(const actqkv_shape& sh, const PagedAttn& p, int32_t* cut) {
  const ChunkCut c = chunk_cut(sh, p);
  cut[0] = kPcRows<1> / c.ks;
  cut[1] = c.ks;
  cut[2] = c.splits;
}
int launch_paged_chunk(const actqkv_shape& sh, const PagedAttn& p, const Workspace& ws, hipStream_t stream) {
  const ChunkCut cut = chunk_cut(sh, p);
  PagedChunk c;
  c.a = p;
  c.tiles = cut.tiles;
  c.splits = cut.splits;
  c.part = ws.scratch_f32();
  c.chosen = PagedBits{nullptr, 0};
  if (sh.head_dim == 64) launch_chunk_ks<64>(cut.ks, c, stream);
  else launch_chunk_ks<128>(cut.ks, c, stream);
  return hip_status("paged attention (chunks)");
}

}  // namespace actqkv
