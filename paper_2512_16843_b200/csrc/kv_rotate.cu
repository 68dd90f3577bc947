// New queries, keys and values of a paged cache: pairs of columns turned by an angle that grows with the row's position,
//   (a, b) -> (a cos - b sin, b cos + a sin),   angle = position * inv_freq[pair],
// queries into their output, keys and values into their pages; or, for whole sequences, queries and keys in their place.
//
// Bound by HBM (128 bytes per row and head each way), by the launch for single tokens.  A warp takes up to 32 heads of one row, so that
// what depends on the row alone (sequence, slot, page, the angles) is found once for 8 KB of data; a lane takes two pieces of
// eight columns that hold both halves of eight pairs, of up to four heads.  Its loads are issued before anything else; the sequence is found
// by all lanes at once, a 32nd of what is left at a time.
//
// Angles: positions reach millions, where an f32 product has lost the angle.  The turns position * inv_freq / 2 pi are formed in f64,
// their fraction is exact there and enough in f32 (2^-25 turns), and sincospif takes it from there.
#include "attn.cuh"
#include "kv_rotate.cuh"

namespace llmc {

namespace {

constexpr uint32_t RO_WARPS = 8;

__device__ __forceinline__ void turn(uint4& lo, uint4& hi, const float2* cs, bool interleaved) {
  uint32_t* w[2] = {&lo.x, &hi.x};
  float a[16];                                       // columns of lo, then of hi
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[p * 8 + 2 * i] = __uint_as_float(w[p][i] << 16);
      a[p * 8 + 2 * i + 1] = __uint_as_float(w[p][i] & 0xFFFF0000u);
    }
  float o[16];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 c = cs[i];
    // pair i: columns (i, i + 8) of the sixteen, or (2 i, 2 i + 1)
    const float xa = interleaved ? a[2 * i] : a[i], xb = interleaved ? a[2 * i + 1] : a[i + 8];
    const float ya = xa * c.x - xb * c.y, yb = xb * c.x + xa * c.y;
    if (interleaved) { o[2 * i] = ya; o[2 * i + 1] = yb; } else { o[i] = ya; o[i + 8] = yb; }
  }
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 v = __floats2bfloat162_rn(o[p * 8 + 2 * i], o[p * 8 + 2 * i + 1]);
      w[p][i] = *reinterpret_cast<const uint32_t*>(&v);
    }
}

// plain load: outputs may take the place of inputs
__device__ __forceinline__ uint4 ld16(const void* p) {
  uint4 v;
  asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}

// the last sequence whose first row is not behind `row`, as seq_of_row finds it, by a whole warp
__device__ __forceinline__ uint32_t seq_of_row_warp(const AttnArgs& a, uint32_t row) {
  const uint32_t lane = threadIdx.x & 31;
  uint32_t lo = 0, hi = a.n_seqs;
  while (hi - lo > 1) {
    const uint32_t step = (hi - lo + 31) / 32, at = lo + lane * step;
    const bool before = lane == 0 || (at < hi && a.cu[at] <= (int32_t)row);
    const uint32_t last = 31 - __clz(__ballot_sync(0xFFFFFFFFu, before));
    lo += last * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

// U: heads of a lane.  PAGED: rows of a paged call; else rows of whole sequences of a.n tokens, keys in their place, values not touched
template <int U, bool PAGED, bool INTERLEAVED>
__global__ void __launch_bounds__(RO_WARPS * 32, 4) k_kv_rotate(const AttnArgs a, const RotateArgs r, uint32_t groups) {
  griddep_sync();
  __shared__ float2 cs[RO_WARPS][32];
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane & 3u;
  const uint32_t q_heads = a.q.ptr ? a.heads : 0u, all_heads = q_heads + (PAGED ? 2 : 1) * a.kv_heads;
  const uint32_t rows = PAGED ? a.n_rows : (uint32_t)min((unsigned long long)a.n_rows, a.n_seqs_dev ? (unsigned long long)*a.n_seqs_dev * a.n : ~0ull);
  // the two pieces of this lane: both halves of the pairs 8 j .. 8 j + 7, or two pieces that stay
  const uint32_t half = r.dims / 16;                  // pieces of the first halves
  const bool turns = j < half;
  const uint32_t pa = INTERLEAVED ? 2 * j : turns ? j : 2 * half + 2 * (j - half), pb = !INTERLEAVED && turns ? j + half : pa + 1;
  const unsigned long long tasks = (unsigned long long)rows * groups;
  for (unsigned long long id = (unsigned long long)blockIdx.x * RO_WARPS + warp; id < tasks; id += (unsigned long long)gridDim.x * RO_WARPS) {
    const uint32_t row = (uint32_t)(id / groups), h0 = (uint32_t)(id % groups) * (8 * U) + (lane >> 2);
    uint4 x[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t h = h0 + u * 8;
      if (h >= all_heads) continue;
      const RowsArgs& src = h < q_heads ? a.q : h < q_heads + a.kv_heads ? a.k : a.v;
      const uint32_t hh = h < q_heads ? h : (h - q_heads) % a.kv_heads;
      const __nv_bfloat16* at = src.ptr + (long long)row * src.tok + (long long)hh * src.head;
      x[u][0] = ld16(at + pa * 8);
      x[u][1] = ld16(at + pb * 8);
    }
    const double freq = lane < r.dims / 2 ? r.inv_freq[lane] : 0.0;
    long long slot, pos;
    uint32_t s = 0;
    int32_t page = -1;
    if (PAGED) {
      s = seq_of_row_warp(a, row);
      const SeqGeo g = seq_geo(a, s);
      if (row < g.row0 || row - g.row0 >= g.all) continue;           // behind the last sequence
      slot = (long long)g.slot0 + (row - g.row0);
      pos = a.first ? (long long)a.first[s] + (row - g.row0) : slot;
      if (slot >= 0) page = page_of(a, s, (uint32_t)slot);
    } else {
      slot = pos = row % a.n;
    }
    __syncwarp();                                     // the last row's angles have been read
    if (lane < r.dims / 2) {
      const double t = (double)pos * freq * 0.15915494309189533577;
      float sn, cn;
      sincospif(2.0f * (float)(t - rint(t)), &sn, &cn);
      cs[warp][lane] = make_float2(cn, sn);
    }
    __syncwarp();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t h = h0 + u * 8;
      if (h >= all_heads) continue;
      const bool is_q = h < q_heads, is_k = !is_q && h < q_heads + a.kv_heads;
      if (turns && (is_q || is_k)) turn(x[u][0], x[u][1], &cs[warp][j * 8], INTERLEAVED);
      const uint32_t hh = is_q ? h : (h - q_heads) % a.kv_heads;
      __nv_bfloat16* to;
      if (is_q) {
        to = a.out.ptr + (long long)row * a.out.tok + (long long)hh * a.out.head;
      } else if (PAGED) {
        if (is_k && j == 0 && a.positions && slot >= 0) a.positions[((size_t)s * a.kv_heads + hh) * a.side_ld + (size_t)slot] = (int32_t)pos;
        if (page < 0) continue;
        to = (is_k ? a.k_pages : a.v_pages) + page_row(a, page, hh, (uint32_t)slot);
      } else {
        to = a.k.ptr + (long long)row * a.k.tok + (long long)hh * a.k.head;
      }
      *reinterpret_cast<uint4*>(to + pa * 8) = x[u][0];
      *reinterpret_cast<uint4*>(to + pb * 8) = x[u][1];
    }
  }
}

}  // namespace

template <int U>
static cudaError_t launch_heads(const AttnArgs& a, const RotateArgs& r, uint32_t heads, cudaStream_t st) {
  const bool paged = a.k_pages != nullptr;
  const uint32_t groups = (heads + 8 * U - 1) / (8 * U);
  // a block for every eight warps' work: with as many as run at a time and a loop, loads and stores of all warps fell into step (32
  // x 1,024 rows of 48 heads: 77 us, 68 so)
  unsigned long long blocks = ((unsigned long long)a.n_rows * groups + RO_WARPS - 1) / RO_WARPS;
  if (blocks > 0x7FFFFFFFull) blocks = 0x7FFFFFFFull;
  auto kern = paged ? (r.interleaved ? k_kv_rotate<U, true, true> : k_kv_rotate<U, true, false>)
                    : (r.interleaved ? k_kv_rotate<U, false, true> : k_kv_rotate<U, false, false>);
  return launch_k(kern, dim3((uint32_t)blocks), dim3(RO_WARPS * 32), 0, st, a, r, groups);
}

cudaError_t launch_kv_rotate(const AttnArgs& a, const RotateArgs& r, int sm_count, cudaStream_t st) {
  if (a.n_rows == 0) return cudaSuccess;
  const uint32_t heads = (a.q.ptr ? a.heads : 0u) + (a.k_pages ? 2 : 1) * a.kv_heads;
  // four heads per lane where that still fills the SMs with warps (32 x 1,024 rows of 48 heads 69.7 -> 65.8 us, of 24 heads 40.2 -> 35.4; a single
  // token of 36 heads takes 3.3 so, 2.7 with two)
  const bool many = heads > 16 && (unsigned long long)a.n_rows * ((heads + 31) / 32) >= 32ull * (uint32_t)sm_count;
  return many ? launch_heads<4>(a, r, heads, st) : launch_heads<2>(a, r, heads, st);
}

}  // namespace llmc
