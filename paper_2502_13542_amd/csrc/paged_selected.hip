// Attention of rows that look at selected pages each (paged_step_body.h has the kernel): a (row, KV head) of its own per group of
// workgroups, its items the halves of the pages in the row's list.
//
// That reads every list, from the L2s and the memory-side cache where rows share pages: 8 to 9 TB/s at best.  Rows of a chunk share most of
// theirs, and where reading every page of the sequence once for a tile of rows takes less, the chunks' kernels do that, with the lists as bits
// (paged_bits.h).  us of lists | so, 32 query and 8 KV heads of 128, 96 pages a row at 100K tokens: 512 rows 2773 | 762 (all pages: 802), 64 391 | 144, 16 132 | 97;
// 8 x 64 rows, 32 pages at 16K 946 | 181; fp32, 8 and 2 heads of 64, 512 rows, 16 pages at 8K 145 | 91.  16 sequences' single tokens at up to 32K, 32 pages each: 49 us = 5.4
// TB/s from memory.
#include "checks.h"
#include "paged_bits.h"
#include "paged_step_body.h"

namespace actqkv {

double paged_chosen_chunk_us(const actqkv_shape& sh, const PagedAttn& p);
double paged_chosen_chunk_f32_us(const actqkv_shape& sh, const PagedAttn& p);
int launch_paged_chosen_chunk(const actqkv_shape& sh, const PagedAttn& p, const PagedBits& bits, const Workspace& ws, hipStream_t stream);
int launch_paged_chosen_chunk_f32(const actqkv_shape& sh, const PagedAttn& p, const PagedBits& bits, const Workspace& ws, hipStream_t stream);

// (At least two wavefronts a SIMD: without the bound fp32 of 128 channels under a cap takes 260 registers, and one.)
template <typename T, int D, int W, bool kCap, bool kBias>
__global__ __launch_bounds__(64 * W, 2) void paged_selected_kernel(PagedStep st) {
  step_body<StepShape<T, D>, T, D, kCap, kBias, true, W>(st);
}
template <typename T, int D, int W>
static void launch_selected_by(const PagedStep& st, hipStream_t stream) {
  const bool cap = st.a.f.cap_in > 0.f, bias = st.a.f.slopes != nullptr;
  const unsigned n = unsigned(st.a.t.n_rows) * st.a.n_kv_heads * st.n_wg;
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(n), dim3(64 * W), 0, stream, st); };
  if (cap && bias) launch(paged_selected_kernel<T, D, W, true, true>);
  else if (cap) launch(paged_selected_kernel<T, D, W, true, false>);
  else if (bias) launch(paged_selected_kernel<T, D, W, false, true>);
  else launch(paged_selected_kernel<T, D, W, false, false>);
}
// A compute unit holds eight wavefronts: with more workgroups than there are compute units two of four side by side, so that one's table, list and merge are
// hidden behind another's keys.  us of eight | two of four: 42 rows, 28 query and 4 KV heads, 4 pages each 20.1 | 16.9, 142 32.6 | 28.9; 32 and 8
// heads, 64 rows of 4 pages 26.8 | 24.1, of 16 91.3 | 90.6, 128 rows of 8 99.0 | 92.4; fewer workgroups: 16 rows of 16 25.6 | 26.6, 1 of 4 7.4 | 8.3.  Of long
// lists only where that fills them: fp32, 8 and 2 heads of 64, 32 pages, 140 rows 114 | 144, 200 rows of 16 87 | 85,
// of 128 140 rows of 8 81 | 73 (under a cap 83 | 75), 200 of 4 48 | 42, of 32 pages, 140 rows 241 | 252; 32 and 8 heads, 64 rows of 4 48 | 42, of 16 211 | 203.
template <typename T, int D>
static void launch_selected(const PagedStep& st, int64_t items, hipStream_t stream) {
  const int64_t wgs = int64_t(st.a.t.n_rows) * st.a.n_kv_heads * st.n_wg;
  if (wgs > kChipCus && (items <= 16 * st.n_wg || 2 * wgs >= 3 * kChipCus)) launch_selected_by<T, D, 4>(st, stream);
  else launch_selected_by<T, D, 8>(st, stream);
}

// The lists as bits: a wavefront a (row, KV head), 64 words and 64 entries at a time.
constexpr int kPbThreads = 256;
__global__ __launch_bounds__(kPbThreads) void paged_bits_kernel(PagedStep st, uint32_t* bits, int words) {
  const PagedTable& t = st.a.t;
  const int lane = threadIdx.x & 63, hk_n = st.a.n_kv_heads;
  const int64_t item = int64_t(blockIdx.x) * (kPbThreads / 64) + (threadIdx.x >> 6);
  if (item >= int64_t(t.n_rows) * hk_n) return;
  const int32_t* idx = st.idx + size_t(item) * st.k_sel;
  const int n = min(max(st.n_sel[item], 0), st.k_sel);
  for (int w0 = 0; w0 < words; w0 += 64) {
    uint32_t word = 0;
    for (int l0 = 0; l0 < n; l0 += 64) {
      const int e = l0 + lane < n ? idx[l0 + lane] : -1;
      for (int j = 0; j < min(n - l0, 64); ++j) {
        const int page = __builtin_amdgcn_readlane(e, j);
        if (page >= 0 && page < t.max_pages && page >> 5 == w0 + lane) word |= 1u << (page & 31);
      }
    }
    if (w0 + lane < words) bits[size_t(item) * words + w0 + lane] = word;
  }
}
constexpr size_t kMostBitBytes = size_t(256) << 20;        // of a call whose lists are taken as bits
static size_t bit_bytes(const actqkv_shape& sh, int n_rows, int max_pages) {
  return size_t(n_rows) * sh.n_kv_heads * ((max_pages + 31) / 32) * sizeof(uint32_t);
}
static size_t chunk_scratch(const actqkv_shape& sh, int batch, int n_rows, int max_new, int max_pages) {
  return align_up(sh.dtype == ACTQKV_F32 ? paged_chunk_f32_scratch_most(sh, batch, n_rows, max_new, max_pages, false)
                                         : paged_chunk_scratch_most(sh, batch, n_rows, max_new, max_pages, false), 256);
}
size_t paged_selected_scratch_most(const actqkv_shape& sh, int batch, int n_rows, int max_new, int max_pages) {
  const size_t parts = step_part_most(sh, int64_t(n_rows) * sh.n_kv_heads);
  if (paged_step_supported(sh, max_new)) return parts;
  return std::max(parts, chunk_scratch(sh, batch, n_rows, max_new, max_pages) +
                             std::min(kMostBitBytes, bit_bytes(sh, n_rows, std::min(max_pages, 32 * kMostBitWords))));
}
// Whether the chunks' kernels take a call: by what they say they take for all pages and 8 us (the bits, their masks), and the lists at 8 TB/s
// and 5 us (for which each row has its own reads and merge to wait for).  us of lists | so: 42 sequences of up to 8 rows at up to 724 tokens, 28 query and 4 KV heads,
// 4 pages each 30 | 24, 24 of them at 1733 tokens 22 | 30; 32 and 8 heads, 1 x 16 rows, 16 pages at 16K 22 | 33, 30 x 10 rows, 2 pages at 300 41 | 16; fp32, 8 and 2 heads
// of 64, 8 x 12 rows, 8 pages at 2K 26 | 26.
bool paged_selected_by_chunks(const actqkv_shape& sh, const PagedAttn& p, int k_sel) {
  if (paged_step_supported(sh, p.t.max_new) || p.t.max_pages > 32 * kMostBitWords ||
      bit_bytes(sh, p.t.n_rows, p.t.max_pages) > kMostBitBytes)
    return false;
  const bool f32 = sh.dtype == ACTQKV_F32;
  const double lists = double(p.t.n_rows) * sh.n_kv_heads * std::min(k_sel, p.t.max_pages) * 2. * kBlock * sh.head_dim * (f32 ? 4. : 2.);
  return (f32 ? paged_chosen_chunk_f32_us(sh, p) : paged_chosen_chunk_us(sh, p)) + 3. < lists / 8e6;
}
int launch_paged_selected(const actqkv_shape& sh, const PagedAttn& p, const int32_t* idx, const int32_t* n_sel, int k_sel,
                          const Workspace& ws, hipStream_t stream) {
  const bool f32 = sh.dtype == ACTQKV_F32;
  const int keys = f32 ? 4096 / sh.head_dim : 64;
  PagedStep st = {};
  st.a = p;
  const int64_t halves = int64_t(std::min(k_sel, p.t.max_pages)) * (kBlock / keys);
  st.n_wg = step_workgroups(int64_t(p.t.n_rows) * sh.n_kv_heads, halves, step_least(keys, sh.head_dim, f32 ? 4 : 2));
  st.part = reinterpret_cast<uint32_t*>(ws.scratch_f32());
  st.counters = ws.counters();
  st.idx = idx;
  st.n_sel = n_sel;
  st.k_sel = k_sel;
  if (paged_selected_by_chunks(sh, p, k_sel)) {
    const PagedTable& t = p.t;
    uint32_t* bits = reinterpret_cast<uint32_t*>(ws.scratch_f32()) + chunk_scratch(sh, t.batch, t.n_rows, t.max_new, t.max_pages) / sizeof(uint32_t);
    const int words = (t.max_pages + 31) / 32;
    const int64_t items = int64_t(t.n_rows) * sh.n_kv_heads;
    hipLaunchKernelGGL(paged_bits_kernel, dim3(unsigned((items + kPbThreads / 64 - 1) / (kPbThreads / 64))), dim3(kPbThreads), 0, stream, st, bits, words);
    ACTQKV_TRY(hip_status("paged attention (selected pages as bits)"));
    return f32 ? launch_paged_chosen_chunk_f32(sh, p, PagedBits{bits, words}, ws, stream)
               : launch_paged_chosen_chunk(sh, p, PagedBits{bits, words}, ws, stream);
  }
  if (f32) {
    if (sh.head_dim == 64) launch_selected<float, 64>(st, halves, stream);
    else launch_selected<float, 128>(st, halves, stream);
  } else {
    if (sh.head_dim == 64) launch_selected<uint16_t, 64>(st, halves, stream);
    else launch_selected<uint16_t, 128>(st, halves, stream);
  }
  return hip_status("paged attention (selected pages)");
}

}  // namespace actqkv
