// Eviction from a paged cache by accumulated attention weight: which tokens stay, and their move to the first slots.
//
// Selection, one workgroup per (sequence, KV head): of the tokens that may go, `need` with the largest weight stay.  The
// weight that the last of them has is found digit by digit (three digits of 11, 11 and 10 bits of the order-preserving integer
// form of a float: a histogram in LDS of the values that share the digits so far); then every wavefront counts what its share
// of the tokens holds above and at that weight and, behind the counts of the wavefronts before it, writes the positions down
// in order.  Equal weights: the lower positions stay.  Integer arithmetic throughout, the same result every time.
//
// Move: the tokens keep their order, so a token never moves up, and slot t of the new cache is filled from a slot >= t.
// In place, a workgroup has a slice of the channels of one (sequence, KV head) to itself and walks the new pages in order: it
// reads everything for some pages, waits, and writes them; nothing that a later step reads lies in them.
#include "paged.h"

namespace actqkv {

constexpr int kEvThreads = 1024, kEvWaves = kEvThreads / 64;
constexpr int kEvBins = 2048;

// Order-preserving integer form: larger weight, larger key; NaN below everything, -0 equal to 0.
__device__ __forceinline__ uint32_t evict_key(float w) {
  if (w != w) return 0u;
  const uint32_t b = __float_as_uint(w + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__global__ __launch_bounds__(kEvThreads) void paged_evict_select_kernel(PagedEvict e) {
  __shared__ uint32_t hist[kEvBins];
  __shared__ uint32_t wave_sum_lds[kEvWaves], found[2];
  __shared__ uint32_t above_lds[kEvWaves], equal_lds[kEvWaves];
  const int hk = blockIdx.x, s = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = paged_tokens(e.t, s);
  int32_t* kept = e.kept + (size_t(s) * e.n_kv_heads + hk) * e.budget;
  const int n_kept = min(n, e.budget);
  if (hk == 0 && tid == 0) e.n_kept[s] = n_kept;
  if (n <= e.budget) {
    for (int i = tid; i < e.budget; i += kEvThreads) kept[i] = i < n ? i : -1;
    return;
  }
  for (int i = tid; i < e.keep_first; i += kEvThreads) kept[i] = i;
  for (int i = tid; i < e.keep_last; i += kEvThreads) kept[e.budget - e.keep_last + i] = n - e.keep_last + i;
  uint32_t need = e.budget - e.keep_first - e.keep_last;
  if (need == 0) return;
  const int lo = e.keep_first, hi = n - e.keep_last;                 // hi - lo > need
  const float* w = e.weights + (size_t(s) * e.n_kv_heads + hk) * e.stride;
  // ---- the key of the last token that stays, digit by digit
  uint32_t prefix = 0, mask = 0;
#pragma unroll 1
  for (int digit = 0; digit < 3; ++digit) {
    const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
    for (int i = tid; i < kEvBins; i += kEvThreads) hist[i] = 0;
    __syncthreads();
    for (int i = lo + tid; i < hi; i += kEvThreads) {
      const uint32_t key = evict_key(w[i]);
      if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & ((1u << bits) - 1u)], 1u);
    }
    __syncthreads();
    // thread i has bins 2 i', 2 i' + 1 from the top down; the bin where the count from the top reaches `need`
    const int top = kEvBins - 1 - 2 * tid;
    const uint32_t h0 = hist[top], h1 = hist[top - 1];
    uint32_t sum = h0 + h1;
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t below = __shfl_up(sum, d, 64);
      if (lane >= d) sum += below;
    }
    if (lane == 63) wave_sum_lds[wave] = sum;
    __syncthreads();
    for (int i = 0; i < wave; ++i) sum += wave_sum_lds[i];
    const uint32_t before = sum - h0 - h1;                          // in bins above this thread's
    if (before < need && need <= sum) {
      const bool second = before + h0 < need;
      found[0] = second ? top - 1 : top;
      found[1] = second ? before + h0 : before;
    }
    __syncthreads();
    prefix |= found[0] << shift;
    mask |= ((1u << bits) - 1u) << shift;
    need -= found[1];
    __syncthreads();
  }
  // ---- positions in order: all above the key, and the first `need` at it
  const int per = ((hi - lo + kEvWaves - 1) / kEvWaves + 63) / 64 * 64;
  const int from = lo + wave * per, to = min(from + per, hi);
  uint32_t above = 0, equal = 0;
  for (int i = from; i < to; i += 64) {
    const uint32_t key = i + lane < to ? evict_key(w[i + lane]) : 0u;
    above += __popcll(__ballot(i + lane < to && key > prefix));
    equal += __popcll(__ballot(i + lane < to && key == prefix));
  }
  if (lane == 0) {
    above_lds[wave] = above;
    equal_lds[wave] = equal;
  }
  __syncthreads();
  uint32_t n_above = 0, n_equal = 0;
  for (int i = 0; i < wave; ++i) {
    n_above += above_lds[i];
    n_equal += equal_lds[i];
  }
  const unsigned long long before = (1ull << lane) - 1;
  for (int i = from; i < to; i += 64) {
    const bool in = i + lane < to;
    const uint32_t key = in ? evict_key(w[i + lane]) : 0u;
    const unsigned long long a = __ballot(in && key > prefix), q = __ballot(in && key == prefix);
    const uint32_t my_above = n_above + __popcll(a & before), my_equal = n_equal + __popcll(q & before);
    if (in && (key > prefix || (key == prefix && my_equal < need)))
      kept[e.keep_first + my_above + min(my_equal, need)] = i + lane;
    n_above += __popcll(a);
    n_equal += __popcll(q);
  }
}

constexpr int kEmThreads = 256;
constexpr int kEmKeyUnits = 4;                    // 16-byte pieces of a key that a workgroup moves
constexpr int kEmRows = 8;                        // channels of the values that a workgroup moves

// Roles of the x dimension: slices of the keys, slices of the values, the weights.  One page a step.
template <typename T, int D>
__global__ __launch_bounds__(kEmThreads) void paged_evict_move_kernel(PagedEvict e) {
  constexpr int V = Vec<T>::N, kKeySlices = D / V / kEmKeyUnits, kValueSlices = D / kEmRows;
  typedef typename Vec<T>::raw raw_t;
  __shared__ size_t from_tile[kBlock];            // page of the token that comes to a slot
  __shared__ int from_slot[kBlock];               // its slot there, -1: none
  const int s = blockIdx.z / e.n_kv_heads, hk = blockIdx.z % e.n_kv_heads, role = blockIdx.x, tid = threadIdx.x;
  const int n = paged_tokens(e.t, s), n_kept = min(n, e.budget);
  const int32_t* kept = e.kept + (size_t(s) * e.n_kv_heads + hk) * e.budget;
  T* kc = static_cast<T*>(e.k_pages);
  T* vc = static_cast<T*>(e.v_pages);
  if (role == kKeySlices + kValueSlices) {        // the weights; zero behind the last token
    if (e.to_weights == nullptr || blockIdx.y != 0) return;
    const size_t row = size_t(s) * e.n_kv_heads + hk;
    const float* w = e.weights + row * e.stride;
    float* to = e.to_weights + row * e.to_stride;
    for (int t0 = 0; t0 < e.to_max_pages * kBlock; t0 += kEmThreads) {
      const int t = t0 + tid;
      const float v = t < n_kept ? w[kept[t]] : 0.f;
      __builtin_amdgcn_s_waitcnt(0);              // read by all before any is written: in place, a slot's own weight goes elsewhere
      __syncthreads();
      if (t < e.to_max_pages * kBlock) to[t] = v;
    }
    return;
  }
  for (int pg = blockIdx.y; pg * kBlock < n_kept; pg += gridDim.y) {
    const int here = min(n_kept - pg * kBlock, kBlock);
    const int page = pg < e.to_max_pages ? e.to_pages[size_t(s) * e.to_max_pages + pg] : -1;
    __syncthreads();
    for (int i = tid; i < kBlock; i += kEmThreads) {
      const int pos = i < here ? kept[pg * kBlock + i] : -1;
      const int from = pos >= 0 ? paged_page(e.t, s, pos / kBlock) : -1;
      from_slot[i] = from >= 0 ? pos % kBlock : -1;
      from_tile[i] = (size_t(max(from, 0)) * e.n_kv_heads + hk) * (kBlock * D);
    }
    __syncthreads();
    if (page < 0 || page >= e.t.n_pages) continue;
    const size_t tile = (size_t(page) * e.n_kv_heads + hk) * (kBlock * D);
    if (role < kKeySlices) {
      constexpr int kEach = kBlock * kEmKeyUnits / kEmThreads;
      raw_t x[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int at = tid + i * kEmThreads, tk = at / kEmKeyUnits, c = role * kEmKeyUnits + at % kEmKeyUnits;
        if (from_slot[tk] >= 0) x[i] = Vec<T>::load_raw(kc + from_tile[tk] + size_t(from_slot[tk]) * D + c * V);
      }
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int at = tid + i * kEmThreads, tk = at / kEmKeyUnits, c = role * kEmKeyUnits + at % kEmKeyUnits;
        if (from_slot[tk] >= 0) *reinterpret_cast<raw_t*>(kc + tile + size_t(tk) * D + c * V) = x[i];
      }
    } else {
      constexpr int kEach = kBlock * kEmRows / kEmThreads;
      T x[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int at = tid + i * kEmThreads, tk = at % kBlock, d = (role - kKeySlices) * kEmRows + at / kBlock;
        if (from_slot[tk] >= 0) x[i] = vc[from_tile[tk] + size_t(d) * kBlock + from_slot[tk]];
      }
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int at = tid + i * kEmThreads, tk = at % kBlock, d = (role - kKeySlices) * kEmRows + at / kBlock;
        if (from_slot[tk] >= 0) vc[tile + size_t(d) * kBlock + tk] = x[i];
      }
    }
  }
}

int launch_paged_evict(const actqkv_shape& sh, const PagedEvict& e, hipStream_t stream) {
  hipLaunchKernelGGL(paged_evict_select_kernel, dim3(sh.n_kv_heads, e.t.batch), dim3(kEvThreads), 0, stream, e);
  const bool in_place = e.to_pages == e.t.pages;
  const int groups = in_place ? 1 : (e.budget + kBlock - 1) / kBlock;
  const int v = sh.dtype == ACTQKV_F32 ? 4 : 8;
  const dim3 grid(sh.head_dim / v / kEmKeyUnits + sh.head_dim / kEmRows + 1, groups, e.t.batch * sh.n_kv_heads);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kEmThreads), 0, stream, e); };
  if (sh.dtype == ACTQKV_F32) {
    if (sh.head_dim == 64) launch(paged_evict_move_kernel<float, 64>);
    else launch(paged_evict_move_kernel<float, 128>);
  } else {
    if (sh.head_dim == 64) launch(paged_evict_move_kernel<uint16_t, 64>);
    else launch(paged_evict_move_kernel<uint16_t, 128>);
  }
  return hip_status("paged evict");
}

}  // namespace actqkv
