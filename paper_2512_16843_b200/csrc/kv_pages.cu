// The paged key/value cache apart from its attention: storing the rows of new tokens, and eviction by received weight.
#include "attn.cuh"
#include "ptx.cuh"

namespace llmc {

namespace {

// ---------------------------------------------------------------------------------------------------------------
// New rows into their pages: a warp takes eight heads of a row, K and V of two heads (32 pieces of 16 bytes) at a time with
// all loads in flight.  What depends on the row alone (its sequence, slot and page) is found once per warp: with a thread
// for every piece that took 28 us for 16,384 rows of 12 heads, 18 as it is (100 MB).  Moves 2 x 128 bytes per row and head each way;
// bound by the launch for a single token, by HBM for a chunk.
// ---------------------------------------------------------------------------------------------------------------
constexpr uint32_t AP_HEADS = 8;
__global__ void __launch_bounds__(256) k_kv_append(const AttnArgs a, uint32_t head_groups) {
  griddep_sync();
  const uint32_t lane = threadIdx.x & 31, part = lane & 15u;
  const unsigned long long tasks = (unsigned long long)a.n_rows * head_groups;
  for (unsigned long long id = (unsigned long long)blockIdx.x * 8 + (threadIdx.x >> 5); id < tasks; id += (unsigned long long)gridDim.x * 8) {
    const uint32_t row = (uint32_t)(id / head_groups), h0 = (uint32_t)(id % head_groups) * AP_HEADS;
    uint4 x[AP_HEADS / 2];
    const RowsArgs& src = part < 8 ? a.k : a.v;
#pragma unroll
    for (uint32_t u = 0; u < AP_HEADS / 2; ++u) {
      const uint32_t hk = h0 + u * 2 + (lane >> 4);
      if (a.k.ptr && hk < a.kv_heads) x[u] = ld_nc16(src.ptr + (long long)row * src.tok + (long long)hk * src.head + (part & 7u) * 8);
    }
    const uint32_t s = seq_of_row(a, row);
    const SeqGeo g = seq_geo(a, s);
    if (row < g.row0 || row - g.row0 >= g.all) continue;             // behind the last sequence
    if (a.zero_rest && row - g.row0 >= g.cnt) {                      // stored, but not computed
      const uint32_t heads = min(AP_HEADS, a.kv_heads - h0) * a.group;
      for (uint32_t i = lane; i < heads * 8; i += 32)
        *reinterpret_cast<uint4*>(a.out.ptr + (long long)row * a.out.tok + (long long)(h0 * a.group + (i >> 3)) * a.out.head + (i & 7u) * 8) = make_uint4(0, 0, 0, 0);
    }
    const long long slot = (long long)g.slot0 + (row - g.row0);
    if (slot < 0) continue;
    if (lane < AP_HEADS && h0 + lane < a.kv_heads) {
      const size_t side = ((size_t)s * a.kv_heads + h0 + lane) * a.side_ld + (size_t)slot;
      if (a.positions) a.positions[side] = a.first ? a.first[s] + (int32_t)(row - g.row0) : (int32_t)slot;
      if (a.weights && a.decay != 0.f) a.weights[side] = 0.f;        // nothing was received there yet
    }
    const int32_t p = a.k.ptr ? page_of(a, s, (uint32_t)slot) : -1;
    if (p < 0) continue;
    __nv_bfloat16* dst = part < 8 ? a.k_pages : a.v_pages;
#pragma unroll
    for (uint32_t u = 0; u < AP_HEADS / 2; ++u) {
      const uint32_t hk = h0 + u * 2 + (lane >> 4);
      if (hk < a.kv_heads) *reinterpret_cast<uint4*>(dst + page_row(a, p, hk, (uint32_t)slot) + (part & 7u) * 8) = x[u];
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------
// Eviction, step 1: one block per (sequence, head) finds the budget-th largest rank by a radix select over 32-bit
// ranks and lists the slots kept in ascending order.
//   rank = 0x7FFFFFFF for protected slots, else the bits of the weight (weights count as >= 0, so their bits order
//   like the numbers)
// Three passes over the 31 bits below the sign.  The first digit has three or four bits of the mantissa, so that weights of
// a few magnitudes spread over many counters.  Ranks are formed once and kept in shared memory where they fit (CACHED), else
// again in every pass; all loads of a round are issued before its stores, which the compiler may not move them across (one
// by one: 47 us instead of 26 for 64 lists of 20,000 to 32,000 slots; four passes of 8 bits without that: 60).  What is left
// are the instructions of 64 blocks, one per list: a block issues in 60 % of its cycles.  Short lists take 256 threads, so
// that several blocks of an SM overlap each other's barriers (768 lists of 400 to 1,500: 28 us with 1024 threads, 13 now).
// ---------------------------------------------------------------------------------------------------------------
constexpr uint32_t EV_CACHED_MAX = 48 * 1024;             // ranks that fit the shared memory of a block
constexpr uint32_t EV_PROTECTED = 0x7FFFFFFFu;             // above the bits of every number
constexpr uint32_t EV_SHORT = 4096;                       // longest list for 256 threads

// sum of x over the warp's earlier lanes
__device__ __forceinline__ uint32_t warp_sum_before(uint32_t x) {
  uint32_t incl = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if ((threadIdx.x & 31) >= (uint32_t)o) incl += y;
  }
  return incl - x;
}

// sum of x over the block's earlier warps (x: one value per warp)
template <uint32_t T>
__device__ __forceinline__ uint32_t warps_sum_before(uint32_t x, uint32_t* warp_sums) {
  const uint32_t lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  __syncthreads();
  if (lane == 0) warp_sums[w] = x;
  __syncthreads();
  return __reduce_add_sync(0xFFFFFFFFu, lane < w ? warp_sums[lane] : 0u);
}

template <bool CACHED, uint32_t T>
__global__ void __launch_bounds__(T, T == 1024 ? 1 : 4) k_evict_select(const EvictArgs a) {
  griddep_sync();
  extern __shared__ __align__(16) uint32_t ranks[];
  constexpr int BITS = T == 1024 ? 12 : 11;               // of the first digit
  constexpr uint32_t BINS = 1u << BITS;
  __shared__ __align__(16) uint32_t hist[BINS], warp_sums[32], pick[2];
  const uint32_t s = blockIdx.x / a.kv_heads, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
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
    for (uint32_t j = keep + threadIdx.x; j < a.budget; j += T) kept_out[j] = -1;
  if (n <= a.budget) {                                    // nothing to drop
    for (uint32_t j = threadIdx.x; j < n; j += T) {
      kept[j] = (int32_t)j;
      if (kept_out) kept_out[j] = (int32_t)j;
    }
    return;
  }
  // largest position of the head
  long long last = (long long)n - 1;
  if (positions) {
    int32_t mx = INT32_MIN;
    for (uint32_t j0 = threadIdx.x; j0 < n; j0 += 8 * T) {
      int32_t v[8];
#pragma unroll
      for (uint32_t u = 0; u < 8; ++u) v[u] = j0 + u * T < n ? __ldg(positions + j0 + u * T) : INT32_MIN;
#pragma unroll
      for (uint32_t u = 0; u < 8; ++u) mx = max(mx, v[u]);
    }
    mx = __reduce_max_sync(0xFFFFFFFFu, mx);
    if (lane == 0) warp_sums[w] = (uint32_t)mx;
    __syncthreads();
    for (uint32_t i = 0; i < T / 32; ++i) mx = max(mx, (int32_t)warp_sums[i]);
    last = mx;
  }
  // protected: position below lo or above hi, in 32 bits.  A position below zero is below any lo, so hi may stop at the
  // lowest number; every position is below a lo beyond the largest one
  const int32_t lo = (int32_t)min(a.sinks, 0x7FFFFFFFu), hi = (int32_t)max(last - (long long)a.recent, (long long)INT32_MIN);
  const bool all = a.sinks > 0x7FFFFFFFu;
  auto rank = [&](float x, int32_t pos) -> uint32_t {
    if (pos < lo || pos > hi || all) return EV_PROTECTED;
    return x > 0.f ? __float_as_uint(x) : 0u;             // not a number and below zero count as zero
  };
  const uint32_t n4 = CACHED ? (n + 3) & ~3u : n;         // the cached list ends in ranks of 0 that are counted out below
  if (CACHED) {
    if (threadIdx.x < n4 - n) ranks[n + threadIdx.x] = 0;
    for (uint32_t j0 = threadIdx.x; j0 < n; j0 += 8 * T) { // all loads of a round before its stores
      float x[8];
      int32_t pos[8];
#pragma unroll
      for (uint32_t u = 0; u < 8; ++u) x[u] = j0 + u * T < n ? __ldg(weights + j0 + u * T) : 0.f;
      if (positions) {
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) pos[u] = j0 + u * T < n ? __ldg(positions + j0 + u * T) : 0;
      } else {
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) pos[u] = (int32_t)(j0 + u * T);
      }
#pragma unroll
      for (uint32_t u = 0; u < 8; ++u)
        if (j0 + u * T < n) ranks[j0 + u * T] = rank(x[u], pos[u]);
    }
  }
  auto four = [&](uint32_t j, uint32_t (&r)[4]) {         // ranks of slots j..j+3 (slots from n on read as 0)
    if (CACHED) {
      const uint4 q = j < n4 ? *reinterpret_cast<const uint4*>(ranks + j) : make_uint4(0, 0, 0, 0);
      r[0] = q.x; r[1] = q.y; r[2] = q.z; r[3] = q.w;
    } else {
#pragma unroll
      for (uint32_t u = 0; u < 4; ++u) r[u] = j + u < n ? rank(weights[j + u], positions ? positions[j + u] : (int32_t)(j + u)) : 0u;
    }
  };
  uint32_t prefix = 0, want = keep;                       // the threshold's leading bits; how many of its group are kept
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int above = pass == 0 ? 31 : pass == 1 ? 31 - BITS : 21 - BITS;
    const int shift = pass == 0 ? 31 - BITS : pass == 1 ? 21 - BITS : 0;
    const uint32_t mask = (1u << (above - shift)) - 1, group = prefix >> above;
    for (uint32_t i = threadIdx.x; i < BINS; i += T) hist[i] = 0;
    __syncthreads();
#pragma unroll 2
    for (uint32_t j = threadIdx.x * 4; j < n; j += 4 * T) {
      uint32_t r[4];
      four(j, r);
#pragma unroll
      for (uint32_t u = 0; u < 4; ++u)
        if (r[u] >> above == group && j + u < n) atomicAdd(&hist[(r[u] >> shift) & mask], 1u);
    }
    __syncthreads();
    // from the largest digit down: the digit in which the want-th largest lies
    constexpr uint32_t PER = BINS / T;
    uint32_t c[PER], sum = 0;
#pragma unroll
    for (uint32_t i = 0; i < PER; ++i) { c[i] = hist[BINS - 1 - (threadIdx.x * PER + i)]; sum += c[i]; }
    uint32_t before = warp_sum_before(sum);
    before += warps_sum_before<T>(__reduce_add_sync(0xFFFFFFFFu, sum), warp_sums);
    if (before < want && want <= before + sum) {
#pragma unroll
      for (uint32_t i = 0; i < PER; ++i) {
        if (before < want && want <= before + c[i]) { pick[0] = BINS - 1 - (threadIdx.x * PER + i); pick[1] = want - before; }
        before += c[i];
      }
    }
    __syncthreads();
    prefix |= pick[0] << shift;
    want = pick[1];
  }
  // prefix is the budget-th largest rank; of the slots that have it the first `want` are kept.  Each warp lists a run of
  // slots, 128 at a time: it counts its run first, and one sum over the warps tells it where its list starts
  const uint32_t run = ((n + T / 32 * 128 - 1) / (T / 32 * 128)) * 128;
  const uint32_t from = min(w * run, n), to = min(from + run, n);
  uint32_t larger = 0, equal = 0;
  for (uint32_t j = from + lane * 4; j < to; j += 128) {
    uint32_t r[4];
    four(j, r);
#pragma unroll
    for (uint32_t u = 0; u < 4; ++u) { larger += r[u] > prefix; equal += r[u] == prefix && j + u < n; }
  }
  larger = warps_sum_before<T>(__reduce_add_sync(0xFFFFFFFFu, larger), warp_sums);
  equal = warps_sum_before<T>(__reduce_add_sync(0xFFFFFFFFu, equal), warp_sums);
  for (uint32_t j0 = from; j0 < to; j0 += 128) {
    const uint32_t j = j0 + lane * 4;
    uint32_t r[4], mine = 0;                              // larger and equal ranks of the lane's four, 16 bits each
    four(j, r);
#pragma unroll
    for (uint32_t u = 0; u < 4; ++u) mine += r[u] > prefix ? 1u : r[u] == prefix && j + u < n ? 0x10000u : 0u;
    const uint32_t at = warp_sum_before(mine), sum = __shfl_sync(0xFFFFFFFFu, at + mine, 31);
    uint32_t gt = larger + (at & 0xFFFFu), eq = equal + (at >> 16);
#pragma unroll
    for (uint32_t u = 0; u < 4; ++u) {
      if (j + u >= n) continue;
      const bool is_gt = r[u] > prefix, is_eq = r[u] == prefix;
      if (is_gt || (is_eq && eq < want)) {
        const uint32_t slot = gt + min(eq, want);
        kept[slot] = (int32_t)(j + u);
        if (kept_out) kept_out[slot] = (int32_t)(j + u);
      }
      gt += is_gt;
      eq += is_eq;
    }
    larger += sum & 0xFFFFu;
    equal += sum >> 16;
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
    go[u] = true;
    x[u] = make_uint4(0, 0, 0, 0);                        // a slot without a page has no row: zeros
    if ((uint32_t)p < a.num_pages)
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
  const uint32_t head_groups = (a.kv_heads + AP_HEADS - 1) / AP_HEADS;
  const unsigned long long tasks = (unsigned long long)a.n_rows * head_groups;
  if (tasks == 0 || a.n_seqs == 0) return cudaSuccess;
  unsigned long long blocks = (tasks + 7) / 8;
  const unsigned long long most = (unsigned long long)sm_count * 16;
  if (blocks > most) blocks = most;
  return launch_k(k_kv_append, dim3((uint32_t)blocks), dim3(256), 0, st, a, head_groups);
}

cudaError_t setup_evict_kernels() {
  return cudaFuncSetAttribute(k_evict_select<true, 1024>, cudaFuncAttributeMaxDynamicSharedMemorySize, EV_CACHED_MAX * 4);
}

cudaError_t launch_evict_tokens(const EvictArgs& a, int sm_count, cudaStream_t st) {
  (void)sm_count;
  if (a.n_seqs == 0) return cudaSuccess;
  const unsigned long long cap = (unsigned long long)a.pages_ld << a.page_shift;
  const uint32_t most = cap < a.max_len ? (uint32_t)cap : a.max_len;
  const dim3 grid(a.n_seqs * a.kv_heads);
  cudaError_t e;
  if (most <= EV_SHORT) e = launch_k(k_evict_select<true, 256>, grid, dim3(256), (most * 4 + 15) & ~15u, st, a);
  else if (most <= EV_CACHED_MAX) e = launch_k(k_evict_select<true, 1024>, grid, dim3(1024), (most * 4 + 15) & ~15u, st, a);
  else e = launch_k(k_evict_select<false, 1024>, grid, dim3(1024), 0, st, a);
  if (e != cudaSuccess) return e;
  return launch_k(k_evict_move, dim3(a.n_seqs * a.kv_heads * ((a.budget + EV_MOVE - 1) / EV_MOVE)), dim3(256), 0, st, a);
}

}  // namespace llmc
