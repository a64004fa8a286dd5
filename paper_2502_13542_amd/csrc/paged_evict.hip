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
// reads everything for some pages, waits, and writes them; nothing that a later step reads lies in them.  A kept token without a page
// moves as zeros: what its new slot held before belongs to nobody.  So there are few workgroups in place, and tokens that stay where they
// are are moved as well: 8 sequences of 8 KV heads of 128 in bf16 from up to 32K tokens to 4096 180 us, to other pages 150; one of 32K 69
// and 43; 8K tokens of 2 heads of 64 in fp32 to 1000 18.5 and 12.5.
#include <type_traits>

#include "paged.h"

namespace actqkv {

constexpr int kEvThreads = 1024, kEvWaves = kEvThreads / 64;
constexpr int kEvBins = 2048;

// Order-preserving integer form: larger weight, larger key; NaN below everything, -0 equal to 0.  0 is of no weight at all: lanes that
// have none take part with it, and since as many tokens as asked for have weights it never is the key of the last.
__device__ __forceinline__ uint32_t evict_key(float w) {
  if (w != w) return 1u;
  const uint32_t b = __float_as_uint(w + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// base + the lanes of `lanes` before this one.
__device__ __forceinline__ uint32_t lanes_below(unsigned long long lanes, uint32_t base) {
  return __builtin_amdgcn_mbcnt_hi(uint32_t(lanes >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(lanes), base));
}

struct EvictLds {
  uint32_t hist[kEvBins];
  uint32_t wave_sum[kEvWaves], found[3];
  uint32_t above[kEvWaves], equal[kEvWaves];
};
// The `need` largest of w[lo .. hi), hi - lo > need > 0, to kept[at ..] in order.  A wavefront has kHold * 64 of them in registers, or (kHold
// 0) reads its share again for every pass, eight words in flight.
template <int kHold>
__device__ __forceinline__ void evict_largest(const float* w, int lo, int hi, uint32_t need, int32_t* kept, EvictLds& l) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = ((hi - lo + kEvWaves - 1) / kEvWaves + 63) / 64 * 64;
  const int from = lo + wave * per, to = min(from + per, hi);
  uint32_t held[kHold > 0 ? kHold : 1];
  if constexpr (kHold > 0) {
    float x[kHold];
#pragma unroll
    for (int k = 0; k < kHold; ++k) x[k] = w[min(from + k * 64 + lane, hi - 1)];
#pragma unroll
    for (int k = 0; k < kHold; ++k) held[k] = from + k * 64 + lane < to ? evict_key(x[k]) : 0u;
  }
  // fn(key, position) for this lane's, 64 neighbours at a time
  auto each = [&](auto fn) {
    if constexpr (kHold > 0) {
#pragma unroll
      for (int k = 0; k < kHold; ++k) {
        if (from + k * 64 < to) fn(held[k], from + k * 64 + lane);
      }
    } else {
      for (int k0 = from; k0 < to; k0 += 8 * 64) {
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = w[min(k0 + k * 64 + lane, to - 1)];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int i = k0 + k * 64 + lane;
          if (k0 + k * 64 < to) fn(i < to ? evict_key(x[k]) : 0u, i);
        }
      }
    }
  };
  // ---- the key of the last token that stays, digit by digit
  uint32_t prefix = 0, mask = 0;
#pragma unroll 1
  for (int digit = 0; digit < 3; ++digit) {
    const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
    for (int i = tid; i < kEvBins; i += kEvThreads) l.hist[i] = 0;
    __syncthreads();
    each([&](uint32_t key, int) {
      if ((key & mask) == prefix) atomicAdd(&l.hist[(key >> shift) & ((1u << bits) - 1u)], 1u);
    });
    __syncthreads();
    // thread i has two bins, from the top down; the bin where the count from the top reaches `need`
    const int top = kEvBins - 1 - 2 * tid;
    const uint32_t h0 = l.hist[top], h1 = l.hist[top - 1];
    uint32_t sum = h0 + h1;
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t below = __shfl_up(sum, d, 64);
      if (lane >= d) sum += below;
    }
    if (lane == 63) l.wave_sum[wave] = sum;
    __syncthreads();
    for (int i = 0; i < wave; ++i) sum += l.wave_sum[i];
    const uint32_t before = sum - h0 - h1;                          // in bins above this thread's
    if (before < need && need <= sum) {
      const bool second = before + h0 < need;
      l.found[0] = second ? top - 1 : top;
      l.found[1] = second ? before + h0 : before;
      l.found[2] = second ? h1 : h0;
    }
    __syncthreads();
    prefix |= l.found[0] << shift;
    mask |= ((1u << bits) - 1u) << shift;
    need -= l.found[1];
    if (need == l.found[2] && prefix != 0) {                        // the whole bin stays: its last need not be known (the lowest bin also counts lanes without a weight)
      prefix -= 1;
      need = 0;
      break;
    }
    __syncthreads();
  }
  // ---- positions in order: all above the key, and the first `need` at it
  uint32_t above = 0, equal = 0;
  each([&](uint32_t key, int) {
    above += __popcll(__ballot(key > prefix));
    equal += __popcll(__ballot(key == prefix));
  });
  if (lane == 0) {
    l.above[wave] = above;
    l.equal[wave] = equal;
  }
  __syncthreads();
  uint32_t n_above = 0, n_equal = 0;
  for (int i = 0; i < wave; ++i) {
    n_above += l.above[i];
    n_equal += l.equal[i];
  }
  each([&](uint32_t key, int i) {
    const unsigned long long a = __ballot(key > prefix), q = __ballot(key == prefix);
    const uint32_t my_above = lanes_below(a, n_above);
    if (q == 0) {                                                    // nearly always
      if (key > prefix) kept[my_above + min(n_equal, need)] = i;
    } else {
      const uint32_t my_equal = lanes_below(q, n_equal);
      if (key > prefix || (key == prefix && my_equal < need)) kept[my_above + min(my_equal, need)] = i;
      n_equal += __popcll(q);
    }
    n_above += __popcll(a);
  });
}

__global__ __launch_bounds__(kEvThreads) void paged_evict_select_kernel(PagedEvict e) {
  __shared__ EvictLds lds;
  const int hk = blockIdx.x, s = blockIdx.y, tid = threadIdx.x;
  const int n = paged_tokens(e.t, s);
  int32_t* kept = e.kept + (size_t(s) * e.n_kv_heads + hk) * e.budget;
  if (hk == 0 && tid == 0) e.n_kept[s] = min(n, e.budget);
  if (n <= e.budget) {
    for (int i = tid; i < e.budget; i += kEvThreads) kept[i] = i < n ? i : -1;
    return;
  }
  for (int i = tid; i < e.keep_first; i += kEvThreads) kept[i] = i;
  for (int i = tid; i < e.keep_last; i += kEvThreads) kept[e.budget - e.keep_last + i] = n - e.keep_last + i;
  const uint32_t need = e.budget - e.keep_first - e.keep_last;
  if (need == 0) return;
  const int lo = e.keep_first, hi = n - e.keep_last;                 // hi - lo > need
  const float* w = e.weights + (size_t(s) * e.n_kv_heads + hk) * e.stride;
  if (hi - lo <= 8 * kEvThreads) evict_largest<8>(w, lo, hi, need, kept + lo, lds);
  else if (hi - lo <= 32 * kEvThreads) evict_largest<32>(w, lo, hi, need, kept + lo, lds);
  else evict_largest<0>(w, lo, hi, need, kept + lo, lds);
}

constexpr int kEmThreads = 256;
constexpr int kEmUnits = 8;                       // 16-byte pieces of a key that a workgroup moves
constexpr int kEmRows = 16;                       // channels of the values that a workgroup moves

// Roles: slices of the keys, slices of the values, the weights.  A step is four pages: 64 KB of keys or half of that
// of values are in flight in a workgroup, which is what a full chip takes (with one page a step 8 sequences to 4096 of up to 32K tokens
// take 160 us instead of 150).
// Values: a thread has two neighbouring slots and reads their values one by one, two bytes each; neighbouring lanes' lie in the same
// few lines, and of a line that holds one kept token all is read.
template <typename T, int D, int kEmPages>
__global__ __launch_bounds__(kEmThreads) void paged_evict_move_kernel(PagedEvict e) {
  constexpr int V = Vec<T>::N, kKeySlices = D / V / kEmUnits, kValueSlices = D / kEmRows;
  typedef typename Vec<T>::raw raw_t;
  typedef std::conditional_t<sizeof(T) == 2, uint32_t, u32x2> pair_t;
  __shared__ int from[kEmPages * kBlock];         // 128 * page + slot of the token that comes to a slot, kNone: no token, kGone: one without a page
  constexpr int kNone = -1, kGone = -2;
  constexpr int kRoles = kKeySlices + kValueSlices + 1;
  const int role = blockIdx.x % kRoles, pair = blockIdx.x / kRoles, s = pair / e.n_kv_heads, hk = pair % e.n_kv_heads, tid = threadIdx.x;
  const int n = paged_tokens(e.t, s), n_kept = min(n, e.budget);
  const int32_t* kept = e.kept + (size_t(s) * e.n_kv_heads + hk) * e.budget;
  T* kc = static_cast<T*>(e.k_pages);
  T* vc = static_cast<T*>(e.v_pages);
  if (role == kKeySlices + kValueSlices) {        // the weights; zero behind the last token
    if (e.to_weights == nullptr || blockIdx.y != 0) return;
    const size_t row = size_t(s) * e.n_kv_heads + hk;
    const float* w = e.weights + row * e.stride;
    float* to = e.to_weights + row * e.to_stride;
    constexpr int kEach = 8;
    for (int t0 = 0; t0 < e.to_max_pages * kBlock; t0 += kEach * kEmThreads) {
      float v[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int t = t0 + i * kEmThreads + tid;
        v[i] = t < n_kept ? w[kept[t]] : 0.f;
      }
      __builtin_amdgcn_s_waitcnt(0);              // read by all before any is written: in place, a slot's own weight goes elsewhere
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int t = t0 + i * kEmThreads + tid;
        if (t < e.to_max_pages * kBlock) to[t] = v[i];
      }
    }
    return;
  }
  if (n <= e.budget && e.to_pages == e.t.pages) return;              // everything is where it belongs
  for (int pg = blockIdx.y * kEmPages; pg * kBlock < n_kept; pg += gridDim.y * kEmPages) {
    int page[kEmPages];
#pragma unroll
    for (int g = 0; g < kEmPages; ++g) {
      const int to = pg + g < e.to_max_pages ? e.to_pages[size_t(s) * e.to_max_pages + pg + g] : -1;
      page[g] = to < e.t.n_pages ? to : -1;
    }
    __syncthreads();
#pragma unroll
    for (int i = tid; i < kEmPages * kBlock; i += kEmThreads) {
      const int t = pg * kBlock + i, pos = t < n_kept ? kept[t] : -1;
      const int at = pos >= 0 ? paged_page(e.t, s, pos / kBlock) : -1;
      from[i] = at >= 0 ? at * kBlock + pos % kBlock : pos >= 0 ? kGone : kNone;
    }
    __syncthreads();
    if (role < kKeySlices) {
      constexpr int kTokens = kEmThreads / kEmUnits, kEach = kBlock / kTokens;
      const int c = (role * kEmUnits + tid % kEmUnits) * V, t0 = tid / kEmUnits;
      raw_t x[kEmPages][kEach];
#pragma unroll
      for (int g = 0; g < kEmPages; ++g)
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          const int src = from[g * kBlock + t0 + i * kTokens];
          x[g][i] = raw_t{};
          if (src >= 0) x[g][i] = Vec<T>::load_raw(kc + ((size_t(src / kBlock) * e.n_kv_heads + hk) * kBlock + src % kBlock) * D + c);
        }
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
#pragma unroll
      for (int g = 0; g < kEmPages; ++g)
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          const int tk = t0 + i * kTokens;
          if (page[g] >= 0 && from[g * kBlock + tk] != kNone)
            *reinterpret_cast<raw_t*>(kc + ((size_t(page[g]) * e.n_kv_heads + hk) * kBlock + tk) * D + c) = x[g][i];
        }
    } else {
      constexpr int kWaves = kEmThreads / 64, kEach = kEmRows / kWaves;
      const int tk = (tid & 63) * 2, d0 = (role - kKeySlices) * kEmRows + (tid >> 6);
      T x[kEmPages][kEach][2];
#pragma unroll
      for (int g = 0; g < kEmPages; ++g)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int src = from[g * kBlock + tk + j];
          const T* at = vc + ((size_t(max(src, 0) / kBlock) * e.n_kv_heads + hk) * D + d0) * kBlock + max(src, 0) % kBlock;
#pragma unroll
          for (int i = 0; i < kEach; ++i) x[g][i][j] = T(0);
          if (src >= 0)
#pragma unroll
            for (int i = 0; i < kEach; ++i) x[g][i][j] = at[i * kWaves * kBlock];
        }
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
#pragma unroll
      for (int g = 0; g < kEmPages; ++g) {
        const bool first = from[g * kBlock + tk] != kNone, second = from[g * kBlock + tk + 1] != kNone;
        T* at = vc + ((size_t(max(page[g], 0)) * e.n_kv_heads + hk) * D + d0) * kBlock + tk;
        if (page[g] < 0) continue;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          T* to = at + i * kWaves * kBlock;
          if (first && second) {
            pair_t both;
            if constexpr (sizeof(T) == 2) both = uint32_t(x[g][i][0]) | uint32_t(x[g][i][1]) << 16;
            else both = u32x2{__float_as_uint(x[g][i][0]), __float_as_uint(x[g][i][1])};
            *reinterpret_cast<pair_t*>(to) = both;
          } else if (first) {
            to[0] = x[g][i][0];
          } else if (second) {
            to[1] = x[g][i][1];
          }
        }
      }
    }
  }
}

int launch_paged_evict(const actqkv_shape& sh, const PagedEvict& e, hipStream_t stream) {
  hipLaunchKernelGGL(paged_evict_select_kernel, dim3(sh.n_kv_heads, e.t.batch), dim3(kEvThreads), 0, stream, e);
  const int v = sh.dtype == ACTQKV_F32 ? 4 : 8;
  const unsigned slices = unsigned(sh.head_dim / v / kEmUnits + sh.head_dim / kEmRows + 1) * e.t.batch * sh.n_kv_heads;
  const int pages = (e.budget + kBlock - 1) / kBlock;
  const bool in_place = e.to_pages == e.t.pages;
  // new pages of a step: four, or one where that leaves compute units idle (in place a workgroup walks all of them): 8K tokens of 2
  // KV heads of 64 in fp32 to 1000, selection included, 16.2 | 13.7 us; 4 sequences 18.4 | 15.7, 16 of 4K 23.0 | 20.8
  const bool single = !in_place && int64_t(slices) * ((pages + 3) / 4) < 2 * kChipCus;
  const dim3 grid(slices, in_place ? 1 : std::min(single ? pages : (pages + 3) / 4, 1024));
  auto launch = [&](auto one, auto four) { hipLaunchKernelGGL(single ? one : four, grid, dim3(kEmThreads), 0, stream, e); };
  if (sh.dtype == ACTQKV_F32) {
    if (sh.head_dim == 64) launch(paged_evict_move_kernel<float, 64, 1>, paged_evict_move_kernel<float, 64, 4>);
    else launch(paged_evict_move_kernel<float, 128, 1>, paged_evict_move_kernel<float, 128, 4>);
  } else {
    if (sh.head_dim == 64) launch(paged_evict_move_kernel<uint16_t, 64, 1>, paged_evict_move_kernel<uint16_t, 64, 4>);
    else launch(paged_evict_move_kernel<uint16_t, 128, 1>, paged_evict_move_kernel<uint16_t, 128, 4>);
  }
  return hip_status("paged evict");
}

}  // namespace actqkv
