// The paged key/value cache apart from its attention: storing the rows of new tokens, and eviction by received weight.
#include "attn.cuh"
#include "ptx.cuh"

namespace llmc {

namespace {

// ---------------------------------------------------------------------------------------------------------------
// New rows into their pages: 16 bytes per thread, eight threads per row of a head (128 bytes: one line), K and V side
// by side.  Moves 2 x 128 bytes per row and head each way; bound by the launch for a single token, by HBM for a chunk.
// ---------------------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256) k_kv_append(const AttnArgs a) {
  griddep_sync();
  const unsigned long long items = (unsigned long long)a.n_rows * a.kv_heads * 16;
  for (unsigned long long id = (unsigned long long)blockIdx.x * 256 + threadIdx.x; id < items; id += (unsigned long long)gridDim.x * 256) {
    const uint32_t part = id & 15u, hk = (uint32_t)((id >> 4) % a.kv_heads), row = (uint32_t)((id >> 4) / a.kv_heads);
    const uint32_t lo = seq_of_row(a, row);
    const SeqGeo g = seq_geo(a, lo);
    if (row < g.row0 || row - g.row0 >= g.cnt) continue;             // behind the last sequence
    const long long slot = (long long)g.slot0 + (row - g.row0);
    if (slot < 0) continue;
    const size_t side = ((size_t)lo * a.kv_heads + hk) * a.side_ld + (size_t)slot;
    if (part == 0 && a.positions) a.positions[side] = a.first ? a.first[lo] + (int32_t)(row - g.row0) : (int32_t)slot;
    if (part == 1 && a.weights && a.decay != 0.f) a.weights[side] = 0.f;          // nothing was received there yet
    if (!a.k.ptr) continue;
    const int32_t p = page_of(a, lo, (uint32_t)slot);
    if (p < 0) continue;
    const RowsArgs& src = part < 8 ? a.k : a.v;
    __nv_bfloat16* dst = (part < 8 ? a.k_pages : a.v_pages) + page_row(a, p, hk, (uint32_t)slot) + (part & 7u) * 8;
    *reinterpret_cast<uint4*>(dst) =
        ld_nc16(src.ptr + (long long)row * src.tok + (long long)hk * src.head + (part & 7u) * 8);
  }
}

// ---------------------------------------------------------------------------------------------------------------
// Eviction, step 1: one block per (sequence, head) finds the budget-th largest rank by a radix select over 32-bit
// ranks (four passes of 8 bits) and lists the slots kept in ascending order.
//   rank = 0xFFFFFFFF for protected slots, else the bits of the weight (weights count as >= 0, so their bits order
//   like the numbers)
// Ranks are computed once and kept in shared memory where they fit (CACHED), else formed again in every pass.
// ---------------------------------------------------------------------------------------------------------------
constexpr uint32_t EV_THREADS = 1024;
constexpr uint32_t EV_CACHED_MAX = 48 * 1024;             // ranks that fit the shared memory of a block

__device__ __forceinline__ uint32_t block_sum_before(uint32_t x, uint32_t* warp_sums, uint32_t& total) {
  // exclusive prefix sum over the block's threads
  const uint32_t lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  uint32_t incl = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= (uint32_t)o) incl += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[w] = incl;
  __syncthreads();
  if (w == 0) {
    uint32_t s = warp_sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, s, o);
      if (lane >= (uint32_t)o) s += y;
    }
    warp_sums[lane] = s;
  }
  __syncthreads();
  total = warp_sums[31];
  return (w ? warp_sums[w - 1] : 0u) + incl - x;
}

template <bool CACHED>
__global__ void __launch_bounds__(EV_THREADS) k_evict_select(const EvictArgs a) {
  griddep_sync();
  extern __shared__ uint32_t ranks[];
  __shared__ uint32_t hist[256], warp_sums[32], pick[4];
  const uint32_t s = blockIdx.x / a.kv_heads;
  const uint32_t cap = min((unsigned long long)a.max_len, (unsigned long long)a.pages_ld << a.page_shift);
  const int32_t raw = a.lens[s];
  const uint32_t n = raw > 0 ? min((uint32_t)raw, cap) : 0u;
  const uint32_t keep = min(n, a.budget);
  int32_t* kept = a.kept + (size_t)blockIdx.x * a.budget;
  int32_t* kept_out = a.kept_out ? a.kept_out + (size_t)blockIdx.x * a.budget : nullptr;
  const float* weights = a.weights + (size_t)blockIdx.x * a.side_ld;
  const int32_t* positions = a.positions ? a.positions + (size_t)blockIdx.x * a.side_ld : nullptr;
  if (blockIdx.x % a.kv_heads == 0 && threadIdx.x == 0) a.count[s] = keep;
  if (kept_out)
    for (uint32_t j = keep + threadIdx.x; j < a.budget; j += EV_THREADS) kept_out[j] = -1;
  if (n <= a.budget) {                                    // nothing to drop
    for (uint32_t j = threadIdx.x; j < n; j += EV_THREADS) {
      kept[j] = (int32_t)j;
      if (kept_out) kept_out[j] = (int32_t)j;
    }
    return;
  }
  // largest position of the head
  long long last = -1;
  if (positions) {
    int32_t mx = INT32_MIN;
    for (uint32_t j = threadIdx.x; j < n; j += EV_THREADS) mx = max(mx, positions[j]);
    for (int o = 16; o > 0; o >>= 1) mx = max(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, o));
    if ((threadIdx.x & 31) == 0) warp_sums[threadIdx.x >> 5] = (uint32_t)mx;
    __syncthreads();
    for (int w = 0; w < 32; ++w) mx = max(mx, (int32_t)warp_sums[w]);
    last = mx;
    __syncthreads();
  } else {
    last = (long long)n - 1;
  }
  auto rank_of = [&](uint32_t j) -> uint32_t {
    const long long pos = positions ? (long long)positions[j] : (long long)j;
    if (pos < (long long)a.sinks || pos > last - (long long)a.recent) return 0xFFFFFFFFu;
    const float w = weights[j];
    return w > 0.f ? __float_as_uint(w) : 0u;             // not a number and below zero count as zero
  };
  uint32_t prefix = 0, want = keep;                       // the threshold's leading bits; how many of its group are kept
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (uint32_t i = threadIdx.x; i < 256; i += EV_THREADS) hist[i] = 0;
    __syncthreads();
    for (uint32_t j = threadIdx.x; j < n; j += EV_THREADS) {
      uint32_t r;
      if (CACHED && shift != 24) r = ranks[j];
      else { r = rank_of(j); if (CACHED) ranks[j] = r; }
      const bool in = shift == 24 || (r >> (shift + 8)) == (prefix >> (shift + 8));
      if (in) atomicAdd(&hist[(r >> shift) & 255u], 1u);
    }
    __syncthreads();
    // from the largest digit down: the digit in which the want-th largest lies
    if (threadIdx.x < 32) {
      uint32_t c[8], sum = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) { c[i] = hist[255 - (threadIdx.x * 8 + i)]; sum += c[i]; }
      uint32_t incl = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (threadIdx.x >= (uint32_t)o) incl += y;
      }
      uint32_t before = incl - sum;
      if (before < want && want <= incl) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (before < want && want <= before + c[i]) { pick[0] = 255 - (threadIdx.x * 8 + i); pick[1] = want - before; }
          before += c[i];
        }
      }
    }
    __syncthreads();
    prefix |= pick[0] << shift;
    want = pick[1];
    __syncthreads();
  }
  // prefix is the budget-th largest rank; of the slots that have it the first `want` are kept
  uint32_t out_base = 0, eq_base = 0;
  for (uint32_t j0 = 0; j0 < n; j0 += EV_THREADS) {
    const uint32_t j = j0 + threadIdx.x;
    const uint32_t r = j < n ? (CACHED ? ranks[j] : rank_of(j)) : 0u;
    const bool eq = j < n && r == prefix;
    uint32_t eq_total, kept_total;
    const uint32_t eq_before = eq_base + block_sum_before(eq ? 1u : 0u, warp_sums, eq_total);
    const bool take = (j < n && r > prefix) || (eq && eq_before < want);
    const uint32_t at = out_base + block_sum_before(take ? 1u : 0u, warp_sums, kept_total);
    if (take) { kept[at] = (int32_t)j; if (kept_out) kept_out[at] = (int32_t)j; }
    eq_base += eq_total;
    out_base += kept_total;
  }
}

// Step 2: the kept rows to their new pages.  Sixteen threads of 16 bytes per entry (K and V), EV_MOVE entries per block.
constexpr uint32_t EV_MOVE = 64;
__global__ void __launch_bounds__(256) k_evict_move(const EvictArgs a) {
  griddep_sync();
  const uint32_t chunks = (a.budget + EV_MOVE - 1) / EV_MOVE;
  const uint32_t c = blockIdx.x % chunks, pair = blockIdx.x / chunks, hk = pair % a.kv_heads, s = pair / a.kv_heads;
  const uint32_t count = a.count[s];
  if (c == 0 && hk == 0 && threadIdx.x == 0) a.new_lens[s] = (int32_t)count;
  const int32_t* kept = a.kept + (size_t)pair * a.budget;
  const uint32_t mask = (1u << a.page_shift) - 1u;
  if (threadIdx.x < EV_MOVE) {
    const uint32_t j = c * EV_MOVE + threadIdx.x;
    if (j < a.budget) {
      const bool real = j < count;
      const size_t src = (size_t)pair * a.side_ld + (real ? (uint32_t)kept[j] : 0u), dst = (size_t)pair * a.new_side_ld + j;
      if (a.new_weights) a.new_weights[dst] = real ? a.weights[src] : 0.f;
      if (a.new_positions) a.new_positions[dst] = real ? (a.positions ? a.positions[src] : kept[j]) : 0;
    }
  }
  const uint32_t part = threadIdx.x & 15u;
  const __nv_bfloat16* from = part < 8 ? a.k_pages : a.v_pages;
  __nv_bfloat16* to = part < 8 ? a.k_pages : a.v_pages;
  constexpr uint32_t U = EV_MOVE / 16;                    // entries per thread, loads of all of them in flight
  uint4 x[U];
  bool go[U];
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    const uint32_t j = c * EV_MOVE + u * 16 + (threadIdx.x >> 4);
    go[u] = false;
    if (j >= count) continue;
    const uint32_t slot = (uint32_t)kept[j];
    const int32_t p = a.pages[(size_t)s * a.pages_ld + (slot >> a.page_shift)];
    if ((uint32_t)p >= a.num_pages) continue;             // a slot without a page has no row to move
    go[u] = true;
    x[u] = ld_stream16(from + (size_t)p * a.page_stride + (((size_t)hk << a.page_shift) + (slot & mask)) * 64 + (part & 7u) * 8);
  }
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    const uint32_t j = c * EV_MOVE + u * 16 + (threadIdx.x >> 4);
    if (!go[u]) continue;
    const int32_t p = a.new_pages[(size_t)s * a.new_pages_ld + (j >> a.page_shift)];
    if ((uint32_t)p >= a.num_pages) continue;
    st_stream16(to + (size_t)p * a.page_stride + (((size_t)hk << a.page_shift) + (j & mask)) * 64 + (part & 7u) * 8, x[u]);
  }
}

}  // namespace

cudaError_t launch_kv_append(const AttnArgs& a, int sm_count, cudaStream_t st) {
  const unsigned long long items = (unsigned long long)a.n_rows * a.kv_heads * 16;
  if (items == 0 || a.n_seqs == 0) return cudaSuccess;
  unsigned long long blocks = (items + 255) / 256;
  const unsigned long long most = (unsigned long long)sm_count * 16;
  if (blocks > most) blocks = most;
  return launch_k(k_kv_append, dim3((uint32_t)blocks), dim3(256), 0, st, a);
}

cudaError_t setup_evict_kernels() {
  return cudaFuncSetAttribute(k_evict_select<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, EV_CACHED_MAX * 4);
}

cudaError_t launch_evict_tokens(const EvictArgs& a, int sm_count, cudaStream_t st) {
  (void)sm_count;
  if (a.n_seqs == 0) return cudaSuccess;
  const unsigned long long cap = (unsigned long long)a.pages_ld << a.page_shift;
  const uint32_t most = cap < a.max_len ? (uint32_t)cap : a.max_len;
  cudaError_t e;
  if (most <= EV_CACHED_MAX)
    e = launch_k(k_evict_select<true>, dim3(a.n_seqs * a.kv_heads), dim3(EV_THREADS), most * 4, st, a);
  else
    e = launch_k(k_evict_select<false>, dim3(a.n_seqs * a.kv_heads), dim3(EV_THREADS), 0, st, a);
  if (e != cudaSuccess) return e;
  return launch_k(k_evict_move, dim3(a.n_seqs * a.kv_heads * ((a.budget + EV_MOVE - 1) / EV_MOVE)), dim3(256), 0, st, a);
}

}  // namespace llmc
