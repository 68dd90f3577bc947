// Attention of few query rows over a paged cache (the next token of every sequence, a handful of drafted ones): up to 16
// rows of a sequence and key/value head, token * group + head of the group.
//
// Such a call reads every cached key and value once (256 bytes per key and head) and computes next to nothing, so its floor is
// HBM, and every SM has to have an even share of the keys.  What bounds it as built is a tile's chain in the four warps (scores,
// maximum, exponentials, product, one tile after the other: some 3 us): the loads in flight would do for twice the rate.  The key tiles of all sequences
// and heads form one list of W tiles of 128 keys, and each of N blocks takes W / N of them in a row (the first W mod N one
// more), whichever sequences they belong to.  A sequence and head that one block has whole is finished there; the others leave their shares
// (sums, maximum, weighted values) in scratch and the block that comes last joins them, in the order of the blocks, so
// that the result does not depend on who was last.
// In a block one warp keeps three tiles of keys and values on their way (TMA, 32 KB each, two blocks per SM: 192 KB in
// flight per SM) and four warps take 32 keys of a tile each, with mma.sync m16n8k16: the 16 rows of the smallest
// tcgen05 shape's 64 or 128 would be all that is used, and there the scores would go through tensor memory for nothing.
// The call's new rows are stored here, too: the block that has the tile they belong to writes them into their page (warp 5)
// and over what was loaded from there (the warp that has these keys; with the stores to memory in the same warp the proxy
// fence behind the change waited for them, 4 us per sequence).
// A sequence's end costs a chain of round trips to memory (the share out, the count, the others' shares); warp 5 takes it,
// and the queries of the next sequence come with its first tile, so that the four warps go on at once.
// Softmax statistics and sums are f32; the weights feed the second product as bf16.
// Measured: one token of 64 sequences of 301 to 4,100 slots, 16 heads on 4, with the scores written: 48 us (147 MB read, 5
// written: 3.2 TB/s); one token behind 516 slots, 12 heads: 12.6 us, launch and the chain load - product - join.
#include <algorithm>
#include "attn_dev.cuh"

namespace llmc {

namespace {

constexpr int FW_THREADS = 192;                              // warps 0-3: products and softmax, 4: loads, 5: joins shares
constexpr uint32_t FW_ST = 3, FW_TILE = 16384, FW_KEYS = 128;
struct FwSmem {
  static constexpr uint32_t K = 0;
  static constexpr uint32_t V = K + FW_ST * FW_TILE;
  static constexpr uint32_t O = V + FW_ST * FW_TILE;         // f32 [warp][row][32]: half of the columns, at the end of a sequence
  static constexpr uint32_t STAT = O + 4 * 16 * 32 * 4;      // f32 [warp][row][2]
  static constexpr uint32_t Q = STAT + 4 * 16 * 2 * 4;       // [2][row][64] bf16: queries of a sequence and head
  static constexpr uint32_t SEG = Q + 2 * 2048;              // FwSeg [2]
  static constexpr uint32_t KMASK = SEG + 128;               // u32 [stage][4]: keys that exist
  static constexpr uint32_t BAR = KMASK + FW_ST * 16;
  static constexpr uint32_t MISC = BAR + 24 * 8;
  static constexpr uint32_t TOTAL = MISC + 32;
};
constexpr uint32_t FW_SMEM = FwSmem::TOTAL + 1024;
static_assert(2 * (FW_SMEM + 1024) <= 233472, "two blocks per SM");

struct FwPlan {
  uint32_t page_box;
  int page_rows, oob_row;
  float* part;                   // [block][2][16][66]
  uint32_t* arrived;             // [n_seqs, kv_heads]: blocks that have left a share; zero between calls
};
constexpr uint32_t FW_SLOT = 16 * 66;

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// key tiles of a sequence: none without rows, else at least one
__device__ __forceinline__ uint32_t seq_tiles(const SeqGeo& g) { return g.cnt ? max(1u, (g.len + FW_KEYS - 1) / FW_KEYS) : 0u; }

// The list of tiles: W in all, block c's share begins at begin(c); `longer` blocks have one more than `each`.
struct FwList {
  uint32_t W, N, each, longer;
  __device__ __forceinline__ uint32_t begin(uint32_t c) const { return c * each + min(c, longer); }
  __device__ __forceinline__ uint32_t block_of(uint32_t t) const {
    const uint32_t in_longer = longer * (each + 1);
    return t < in_longer ? t / (each + 1) : longer + (t - in_longer) / each;
  }
};
// A sequence and head in it: first = number of its tile 0 of nt.
struct FwPlace { uint32_t s, hk, nt, first; SeqGeo g; };
// What the load warp tells the others about it: tiles j0 .. j1 - 1 are this block's; nt == 0: there is no more.
struct FwSeg { FwPlace at; uint32_t j0, j1; int32_t pos0; };
static_assert(sizeof(FwSeg) <= 64, "two fit their place in shared memory");

__device__ __forceinline__ uint32_t warp_scan(uint32_t x) {  // inclusive sum over the lanes
  const uint32_t lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, x, o);
    if (lane >= (uint32_t)o) x += y;
  }
  return x;
}
// The list, and the place of its tile number begin(block) (one warp together).
__device__ __noinline__ void find_place(const AttnArgs& a, uint32_t block, uint32_t blocks, FwList& L, FwPlace& p) {
  const uint32_t lane = threadIdx.x & 31;
  uint32_t sum = 0, kept = 0;
#pragma unroll 1
  for (uint32_t s0 = 0; s0 < a.n_seqs; s0 += 32) {
    kept = s0 + lane < a.n_seqs ? seq_tiles(seq_geo(a, s0 + lane)) * a.kv_heads : 0u;
    sum += kept;
  }
  L.W = __reduce_add_sync(0xFFFFFFFFu, sum);
  L.N = min(blocks, L.W);                                    // blocks with work
  L.each = L.N ? L.W / L.N : 0u;
  L.longer = L.W - L.N * L.each;
  if (block >= L.N) return;
  const uint32_t t = L.begin(block);
  uint32_t before = 0;
#pragma unroll 1
  for (uint32_t s0 = 0; s0 < a.n_seqs; s0 += 32) {
    const uint32_t mine = a.n_seqs <= 32 ? kept : s0 + lane < a.n_seqs ? seq_tiles(seq_geo(a, s0 + lane)) * a.kv_heads : 0u;
    const uint32_t incl = warp_scan(mine);
    const uint32_t hit = __ballot_sync(0xFFFFFFFFu, before + incl > t);
    if (hit) {
      const int l = __ffs(hit) - 1;
      p.s = s0 + l;
      before += __shfl_sync(0xFFFFFFFFu, incl - mine, l);
      break;
    }
    before += __shfl_sync(0xFFFFFFFFu, incl, 31);
  }
  p.g = seq_geo(a, p.s);
  p.nt = seq_tiles(p.g);
  p.hk = (t - before) / p.nt;
  p.first = before + p.hk * p.nt;
}
// eight columns of a finished row
__device__ __noinline__ void few_output(const AttnArgs& a, const FwPlace& at, uint32_t R, uint32_t c0, float mx, float lt, const float (&x)[8]) {
  const uint32_t token = R / a.group, h = at.hk * a.group + R % a.group;
  const bool dead = lt == 0.f;                               // nothing seen
  const float inv = dead ? 0.f : 1.f / lt;
  uint32_t w[4];
#pragma unroll
  for (uint32_t y = 0; y < 4; ++y) w[y] = pack2(dead ? 0.f : x[2 * y] * inv, dead ? 0.f : x[2 * y + 1] * inv);
  const size_t row = (size_t)at.g.row0 + token;
  *reinterpret_cast<uint4*>(a.out.ptr + (long long)row * a.out.tok + (long long)h * a.out.head + c0) = make_uint4(w[0], w[1], w[2], w[3]);
  if (a.lse && c0 == 0) a.lse[row * a.heads + h] = dead ? -INFINITY : log_sum(mx, lt);
  if (a.stat && c0 == 0) a.stat[row * a.heads + h] = make_float2(mx, lt);
}
// One of the 16-byte pieces of the new row of a slot: eight lanes have its key, eight its value.
__device__ __forceinline__ uint4 new_piece(const AttnArgs& a, const FwPlace& at, uint32_t slot) {
  const uint32_t part = threadIdx.x & 15u;
  const RowsArgs& src = part < 8 ? a.k : a.v;
  return ld_nc16(src.ptr + (long long)(at.g.row0 + (uint32_t)((int32_t)slot - at.g.slot0)) * src.tok + (long long)at.hk * src.head + (part & 7u) * 8);
}
// The new rows with slots from .. to - 1: into their pages and the side arrays (one warp, two rows at a time).
__device__ __noinline__ void store_new(const AttnArgs& a, const FwPlace& at, uint32_t from, uint32_t to) {
  const uint32_t lane = threadIdx.x & 31, part = lane & 15u;
#pragma unroll 1
  for (uint32_t slot = from + (lane >> 4); slot < to; slot += 2) {
    const size_t side = ((size_t)at.s * a.kv_heads + at.hk) * a.side_ld + slot;
    const int32_t i = (int32_t)slot - at.g.slot0;
    if (part == 0 && a.positions) a.positions[side] = a.first ? a.first[at.s] + i : (int32_t)slot;
    if (part == 1 && a.weights && a.decay != 0.f) a.weights[side] = 0.f;
    if (!a.k.ptr) continue;
    const uint4 v = new_piece(a, at, slot);
    const int32_t pg = page_of(a, at.s, slot);
    if (pg >= 0) *reinterpret_cast<uint4*>((part < 8 ? a.k_pages : a.v_pages) + page_row(a, pg, at.hk, slot) + (part & 7u) * 8) = v;
  }
}
// Zeros for the rows that are not computed, in the heads of one key/value head (one warp).
__device__ __noinline__ void zero_rest(const AttnArgs& a, const FwPlace& at) {
  const unsigned long long pieces = (unsigned long long)(at.g.all - at.g.cnt) * a.group * 8;
#pragma unroll 1
  for (unsigned long long i = threadIdx.x & 31; i < pieces; i += 32) {
    const uint32_t R = (uint32_t)(i >> 3), token = at.g.cnt + R / a.group, h = at.hk * a.group + R % a.group;
    *reinterpret_cast<uint4*>(a.out.ptr + (long long)(at.g.row0 + token) * a.out.tok + (long long)h * a.out.head + (i & 7u) * 8) = make_uint4(0, 0, 0, 0);
  }
}
__device__ __noinline__ void next_place(const AttnArgs& a, FwPlace& p) {
  p.first += p.nt;
  if (++p.hk < a.kv_heads) return;
  p.hk = 0;
  do {
    if (++p.s >= a.n_seqs) { p.nt = 0; return; }
    p.g = seq_geo(a, p.s);
    p.nt = seq_tiles(p.g);
  } while (!p.nt);
}

}  // namespace

template <bool MOD>
__global__ void __launch_bounds__(FW_THREADS, 2)
k_attn_few(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
           const __grid_constant__ AttnArgs a, const __grid_constant__ FwPlan p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gbase = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bar0 = base + FwSmem::BAR;
  auto full = [&](uint32_t s) { return bar0 + 8 * s; };
  auto empty = [&](uint32_t s) { return bar0 + 8 * (FW_ST + s); };
  const uint32_t together = bar0 + 8 * 2 * FW_ST;
  auto share_out = [&](uint32_t b) { return together + 48 + 8 * b; };      // each completes once at most
  auto seg_full = [&](uint32_t b) { return together + 16 + 8 * b; };
  auto seg_empty = [&](uint32_t b) { return together + 32 + 8 * b; };
  FwSeg* segs = reinterpret_cast<FwSeg*>(gbase + FwSmem::SEG);
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(gbase + FwSmem::MISC);
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < FW_ST; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 4); }
    mbar_init(together, 4);
    for (uint32_t b = 0; b < 2; ++b) {
      mbar_init(share_out(b), 4); mbar_init(seg_full(b), 1); mbar_init(seg_empty(b), 4 + 1);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  griddep_sync();
  const unsigned long long lim = wait_limit(a.status);

  if (warp == 4) {
    // ---------------------------------------------------------------- loads
    FwList L;
    FwPlace at;
    find_place(a, blockIdx.x, gridDim.x, L, at);
    const bool work = blockIdx.x < L.N && !producer_idle(a.status);
    const uint32_t t0 = work ? L.begin(blockIdx.x) : 0u, t1 = work ? L.begin(blockIdx.x + 1) : 0u;
    bool ok = true;
    uint32_t e = 0, n = 0;
#pragma unroll 1
    for (uint32_t t = t0;;) {
      const bool end = t >= t1;
      if (end && producer_idle(a.status)) break;
      const uint32_t j0 = end ? 0u : t - at.first, j1 = end ? 0u : min(at.nt, t1 - at.first), b = n & 1u;
      ok = warp_wait(seg_empty(b), ((n >> 1) & 1u) ^ 1u, abort_flag, lim, 32);
      if (!ok) break;
      if (end) at.nt = 0;
#pragma unroll 1
      for (uint32_t j = j0; j <= j1 && ok; ++j) {
        if (j < j1) {
          const uint32_t s = e % FW_ST, boxes = FW_KEYS / p.page_box, per_word = max(1u, 32u / p.page_box);
          int row = p.oob_row;
          if (lane < boxes) {
            const uint32_t slot = j * FW_KEYS + lane * p.page_box;
            const int32_t pg = slot < at.g.len ? page_of(a, at.s, slot) : -1;
            if (pg >= 0) row = pg * p.page_rows + (int)((at.hk << a.page_shift) + (slot & ((1u << a.page_shift) - 1u)));
          }
          const uint32_t exist = __ballot_sync(0xFFFFFFFFu, row != p.oob_row);
          ok = warp_wait(empty(s), ((e / FW_ST) & 1u) ^ 1u, abort_flag, lim, 32);
          if (!ok) break;
          if (lane < 4) {
            // 32 keys: part of one box, one box, or two boxes of 16
            uint32_t word = 0;
            if (p.page_box >= 32) word = (exist >> (lane * 32 / p.page_box)) & 1u ? ~0u : 0u;
            else for (uint32_t x = 0; x < per_word; ++x) word |= (exist >> (lane * per_word + x)) & 1u ? 0xFFFFu << (16 * x) : 0u;
            reinterpret_cast<volatile uint32_t*>(gbase + FwSmem::KMASK)[s * 4 + lane] = word;
          }
          __syncwarp();
          if (lane == 0) mbar_expect_tx(full(s), 2 * FW_TILE);
          __syncwarp();
          if (lane < boxes) {
            const uint32_t off = s * FW_TILE + lane * p.page_box * 128;
            tma_load_2d(base + FwSmem::K + off, &map_k, 0, row, full(s));
            tma_load_2d(base + FwSmem::V + off, &map_v, 0, row, full(s));
          }
          ++e;
        }
        if (j == j0) {
          // behind the first tile's loads: the queries (zeros in rows that do not exist), then the description
          const uint32_t rows = end ? 0u : at.g.cnt * a.group;
#pragma unroll
          for (uint32_t u = 0; u < 4; ++u) {
            const uint32_t R = u * 4 + (lane >> 3), c = lane & 7u;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (R < rows)
              v = ld_nc16(a.q.ptr + (long long)(at.g.row0 + R / a.group) * a.q.tok + (long long)(at.hk * a.group + R % a.group) * a.q.head + c * 8);
            *reinterpret_cast<uint4*>(gbase + FwSmem::Q + b * 2048 + R * 128 + ((c ^ (R & 7u)) << 4)) = v;
          }
          if (lane == 0) segs[b] = FwSeg{at, j0, j1, end ? 0 : a.first ? a.first[at.s] : at.g.slot0};
          __syncwarp();
          if (lane == 0) mbar_arrive(seg_full(b));
        }
      }
      if (!ok || end) break;
      ++n;
      t = at.first + j1;
      if (t < t1) next_place(a, at);
    }
    if (!ok && lane == 0) { *abort_flag = 1; atomicExch(a.status, 1u); }
    __syncwarp();
    if (lane == 0 && *abort_flag) {                          // loads in flight must land before shared memory is released
      volatile uint32_t never = 0;
#pragma unroll 1
      for (uint32_t b = 0; b < FW_ST && b < e; ++b) mbar_wait(full((e - 1 - b) % FW_ST), ((e - 1 - b) / FW_ST) & 1u, &never, 200000000ull);
    }
  } else if (warp == 5) {
    // ---------------------------------------------------------------- shares of sequences that several blocks work on
    FwList L;
    FwPlace unused;
    find_place(a, blockIdx.x, gridDim.x, L, unused);
    const bool fresh = a.k.ptr || a.positions || (a.weights && a.decay != 0.f);
    bool ok = true;
#pragma unroll 1
    for (uint32_t n = 0;; ++n) {
      ok = warp_wait(seg_full(n & 1u), (n >> 1) & 1u, abort_flag, lim, 64);
      if (!ok) break;
      const FwSeg seg = segs[n & 1u];
      const FwPlace& at = seg.at;
      if (!at.nt) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(seg_empty(n & 1u));
      if (fresh) {
        const uint32_t from = (uint32_t)max(at.g.slot0, (int32_t)(seg.j0 * FW_KEYS));
        const uint32_t to = min(min(at.g.len, seg.j1 * FW_KEYS), (uint32_t)max(0, at.g.slot0 + (int32_t)at.g.all));
        if (from < to) store_new(a, at, from, to);
        __syncwarp();
      }
      if (a.zero_rest && seg.j0 == 0) zero_rest(a, at);
      if (seg.j0 == 0 && seg.j1 == at.nt) continue;
      ok = warp_wait(share_out(seg.j0 == 0 ? 1u : 0u), 0u, abort_flag, lim, 64);
      if (!ok) break;
      const uint32_t c_lo = L.block_of(at.first), c_hi = L.block_of(at.first + at.nt - 1);
      uint32_t last = 0;
      if (lane == 0) {
        __threadfence();                                     // the block's share before its count (the barrier orders it before this)
        uint32_t* count = p.arrived + (size_t)at.s * a.kv_heads + at.hk;
        last = atomicAdd(count, 1u) == c_hi - c_lo ? 1u : 0u;
        if (last) *count = 0;                                // for the next call
        __threadfence();
      }
      last = __shfl_sync(0xFFFFFFFFu, last, 0);
      if (!last) continue;
      // four rows at a time, eight lanes (of eight columns) each
#pragma unroll 1
      for (uint32_t R = lane >> 3; R < at.g.cnt * a.group; R += 4) {
        const uint32_t c0 = (lane & 7u) * 8;
        auto share = [&](uint32_t b) { return p.part + ((size_t)b * 2 + (b == c_lo ? 1 : 0)) * FW_SLOT; };
        float mx = -INFINITY, lt = 0.f, x[8];
#pragma unroll
        for (uint32_t y = 0; y < 8; ++y) x[y] = 0.f;
        float2 ml_n = __ldcg(reinterpret_cast<const float2*>(share(c_lo) + 1024 + R * 2));
        float4 v0_n = __ldcg(reinterpret_cast<const float4*>(share(c_lo) + R * 64 + c0)), v1_n = __ldcg(reinterpret_cast<const float4*>(share(c_lo) + R * 64 + c0 + 4));
#pragma unroll 1
        for (uint32_t b = c_lo; b <= c_hi; ++b) {
          const float2 ml = ml_n;
          const float v[8] = {v0_n.x, v0_n.y, v0_n.z, v0_n.w, v1_n.x, v1_n.y, v1_n.z, v1_n.w};
          if (b < c_hi) {                                    // the next share is on its way
            ml_n = __ldcg(reinterpret_cast<const float2*>(share(b + 1) + 1024 + R * 2));
            v0_n = __ldcg(reinterpret_cast<const float4*>(share(b + 1) + R * 64 + c0));
            v1_n = __ldcg(reinterpret_cast<const float4*>(share(b + 1) + R * 64 + c0 + 4));
          }
          if (ml.y == 0.f) continue;                         // nothing seen in this share
          const float m_new = fmaxf(mx, ml.x), f0 = ex2f(mx - m_new), f = ex2f(ml.x - m_new);
#pragma unroll
          for (uint32_t y = 0; y < 8; ++y) x[y] = fmaf(v[y], f, mx == -INFINITY ? 0.f : x[y] * f0);
          lt = fmaf(ml.y, f, mx == -INFINITY ? 0.f : lt * f0);
          mx = m_new;
        }
        few_output(a, at, R, c0, mx, lt, x);
      }
      __syncwarp();
    }
    if (!ok && lane == 0) { *abort_flag = 1; atomicExch(a.status, 1u); }
  } else {
    // ---------------------------------------------------------------- products and softmax: 32 keys of a tile per warp
    const uint32_t quad = lane >> 2, pair = (lane & 3u) * 2; // rows quad and quad + 8, columns pair and pair + 1 of every 8
    const float sc = a.m.scale * LOG2E_F;
    bool ok = true;
    uint32_t e = 0, n_meet = 0;
    auto meet = [&]() -> bool {
      __syncwarp();
      if (lane == 0) mbar_arrive(together);
      const bool met = warp_wait(together, n_meet & 1u, abort_flag, lim, 0);
      ++n_meet;
      return met;
    };
#pragma unroll 1
    for (uint32_t n = 0;; ++n) {
      ok = warp_wait(seg_full(n & 1u), (n >> 1) & 1u, abort_flag, lim, 32);
      if (!ok) break;
      const FwSeg seg = segs[n & 1u];
      const FwPlace& at = seg.at;
      if (!at.nt) break;
      const uint32_t j0 = seg.j0, j1 = seg.j1, rows = at.g.cnt * a.group;
      const uint32_t new_end = min(at.g.len, (uint32_t)max(0, at.g.slot0 + (int32_t)at.g.all));      // behind the last new row's slot
      const int32_t pos0 = seg.pos0;
      uint32_t qf[4][4];
#pragma unroll
      for (uint32_t kk = 0; kk < 4; ++kk) {
        const uint32_t R = lane & 15u;
        ldsm4(base + FwSmem::Q + (n & 1u) * 2048 + R * 128 + (((kk * 2 + (lane >> 4)) ^ (R & 7u)) << 4), qf[kk]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(seg_empty(n & 1u));
      // the two rows of this thread
      int32_t hi[2], qpos[2];
      float slope[2] = {0.f, 0.f};
      const float* table[2] = {nullptr, nullptr};
#pragma unroll
      for (uint32_t u = 0; u < 2; ++u) {
        const uint32_t R = quad + u * 8;
        const bool mine = R < rows;
        const uint32_t token = mine ? R / a.group : 0u, h = at.hk * a.group + (mine ? R % a.group : 0u);
        hi[u] = !mine ? 0 : a.m.causal ? min(at.g.slot0 + (int32_t)token + 1, (int32_t)at.g.len) : (int32_t)at.g.len;
        qpos[u] = pos0 + (int32_t)token;
        if (MOD && a.m.slopes) slope[u] = a.m.slopes[h] * LOG2E_F;
        if (MOD && a.m.table) table[u] = a.m.table + (size_t)h * (2 * a.m.reach + 1) + a.m.reach;
      }
      const int32_t* positions = MOD && a.positions ? a.positions + ((size_t)at.s * a.kv_heads + at.hk) * a.side_ld : nullptr;
      auto key_pos = [&](uint32_t key) -> int32_t {          // (a new row's position follows from its slot: it is being written)
        return (int32_t)key >= at.g.slot0 ? pos0 + ((int32_t)key - at.g.slot0) : positions && key < at.g.len ? positions[key] : (int32_t)key;
      };
      float o[8][4];
#pragma unroll
      for (uint32_t x = 0; x < 8; ++x) o[x][0] = o[x][1] = o[x][2] = o[x][3] = 0.f;
      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll 1
      for (uint32_t j = j0; j < j1; ++j, ++e) {
        const uint32_t s = e % FW_ST, k0 = j * FW_KEYS + warp * 32;
        // new rows among this warp's keys replace what TMA reads of their (not yet written) places
        const uint32_t new0 = (uint32_t)max(at.g.slot0, (int32_t)k0) + (lane >> 4), new1 = min(k0 + 32, new_end);
        const bool news = a.k.ptr && (int32_t)(k0 + 32) > at.g.slot0 && k0 < new_end;
        uint4 piece = make_uint4(0, 0, 0, 0);
        if (news && new0 < new1) piece = new_piece(a, at, new0);
        ok = warp_wait(full(s), (e / FW_ST) & 1u, abort_flag, lim, 32);
        if (!ok) break;
        const uint32_t exist = reinterpret_cast<volatile const uint32_t*>(gbase + FwSmem::KMASK)[s * 4 + warp];
        if (news) {
          uint8_t* tile = gbase + ((lane & 15u) < 8 ? FwSmem::K : FwSmem::V) + s * FW_TILE;
#pragma unroll 1
          for (uint32_t slot = new0; slot < new1; slot += 2) {
            const uint32_t r = slot - j * FW_KEYS;
            *reinterpret_cast<uint4*>(tile + r * 128 + (((lane & 7u) ^ (r & 7u)) << 4)) = piece;
            if (slot + 2 < new1) piece = new_piece(a, at, slot + 2);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");    // (the next tile there comes by TMA)
          __syncwarp();
        }
        if (k0 < at.g.len) {
          // S = Q K^T: four blocks of eight keys
          float c[4][4];
#pragma unroll
          for (uint32_t n = 0; n < 4; ++n) c[n][0] = c[n][1] = c[n][2] = c[n][3] = 0.f;
#pragma unroll
          for (uint32_t half = 0; half < 2; ++half) {
            uint32_t b[4][4];
#pragma unroll
            for (uint32_t n = 0; n < 4; ++n) {
              const uint32_t key = warp * 32 + n * 8 + (lane & 7u);
              ldsm4(base + FwSmem::K + s * FW_TILE + key * 128 + (((half * 4 + (lane >> 3)) ^ (key & 7u)) << 4), b[n]);
            }
#pragma unroll
            for (uint32_t n = 0; n < 4; ++n) mma16816(c[n], qf[half * 2], b[n][0], b[n][1]);
#pragma unroll
            for (uint32_t n = 0; n < 4; ++n) mma16816(c[n], qf[half * 2 + 1], b[n][2], b[n][3]);
          }
          // scores in base-2 units, masked
          if (MOD) {
#pragma unroll
            for (uint32_t n = 0; n < 4; ++n) {
#pragma unroll
              for (uint32_t x = 0; x < 4; ++x) c[n][x] *= a.m.cap > 0.f ? a.m.scale / a.m.cap : sc;
            }
            if (a.m.cap > 0.f) {
#pragma unroll
              for (uint32_t n = 0; n < 4; ++n) {
#pragma unroll
                for (uint32_t x = 0; x < 4; ++x)
                  c[n][x] = (fabsf(c[n][x]) <= 0.75f ? f2_lo(tanh_small2(f2_dup(c[n][x]))) : tanh_large(c[n][x])) * (a.m.cap * LOG2E_F);
              }
            }
            if (a.m.slopes || a.m.table) {
#pragma unroll
              for (uint32_t n = 0; n < 4; ++n) {
#pragma unroll
                for (uint32_t y = 0; y < 2; ++y) {
                  const uint32_t key = k0 + n * 8 + pair + y;
                  const int32_t kpos = key_pos(key);
#pragma unroll
                  for (uint32_t u = 0; u < 2; ++u) {
                    const int32_t d = kpos - qpos[u];
                    float z = fmaf(-slope[u], fabsf((float)d), c[n][u * 2 + y]);
                    if (a.m.table) {
                      const float b = __ldg(table[u] + min(max(d, -a.m.reach), a.m.reach));
                      z = b == -INFINITY ? b : z + entry2(b);
                    }
                    c[n][u * 2 + y] = z;
                  }
                }
              }
            }
          } else {
#pragma unroll
            for (uint32_t n = 0; n < 4; ++n) {
#pragma unroll
              for (uint32_t x = 0; x < 4; ++x) c[n][x] *= sc;
            }
          }
          float mt[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (uint32_t n = 0; n < 4; ++n) {
#pragma unroll
            for (uint32_t x = 0; x < 4; ++x) {
              const uint32_t in = n * 8 + pair + (x & 1u);
              const bool see = (int32_t)(k0 + in) < hi[x >> 1] && ((exist >> in) & 1u);
              c[n][x] = see ? c[n][x] : -INFINITY;
              mt[x >> 1] = fmaxf(mt[x >> 1], c[n][x]);
            }
          }
          if (a.scores) {
            // for the received weights: 16 rows * 4 bytes per key at most, against 256 that were read
#pragma unroll
            for (uint32_t u = 0; u < 2; ++u) {
              const uint32_t R = quad + u * 8;
              if (R >= rows) continue;
              float* dst = a.scores + (((size_t)at.s * a.kv_heads + at.hk) * a.score_rows + R) * a.score_ld + k0 + pair;
#pragma unroll
              for (uint32_t n = 0; n < 4; ++n) *reinterpret_cast<float2*>(dst + n * 8) = make_float2(c[n][u * 2], c[n][u * 2 + 1]);
            }
          }
          float nm[2];
#pragma unroll
          for (uint32_t u = 0; u < 2; ++u) {
            mt[u] = fmaxf(mt[u], __shfl_xor_sync(0xFFFFFFFFu, mt[u], 1));
            mt[u] = fmaxf(mt[u], __shfl_xor_sync(0xFFFFFFFFu, mt[u], 2));
            const float m_new = fmaxf(m[u], mt[u]);
            const float corr = m_new == -INFINITY ? 1.f : ex2f(m[u] - m_new);
            m[u] = m_new;
            nm[u] = m_new == -INFINITY ? 0.f : -m_new;
            l[u] *= corr;
#pragma unroll
            for (uint32_t x = 0; x < 8; ++x) { o[x][u * 2] *= corr; o[x][u * 2 + 1] *= corr; }
          }
          // P and its sums
          uint32_t pa[2][4];
#pragma unroll
          for (uint32_t g = 0; g < 2; ++g) {
#pragma unroll
            for (uint32_t y = 0; y < 2; ++y) {
#pragma unroll
              for (uint32_t u = 0; u < 2; ++u) {
                const float p0 = ex2f(c[g * 2 + y][u * 2] + nm[u]), p1 = ex2f(c[g * 2 + y][u * 2 + 1] + nm[u]);
                l[u] += p0 + p1;
                pa[g][y * 2 + u] = pack2(p0, p1);
              }
            }
          }
          // O += P V, 16 keys at a time (one copy of the code)
#pragma unroll 1
          for (uint32_t g = 0; g < 2; ++g) {
            uint32_t pg[4];
#pragma unroll
            for (uint32_t y = 0; y < 4; ++y) pg[y] = g ? pa[1][y] : pa[0][y];
            const uint32_t key = warp * 32 + g * 16 + (lane & 15u), row = base + FwSmem::V + s * FW_TILE + key * 128;
            uint32_t vb[4][4], acc = 0;
#pragma unroll
            for (uint32_t x = 0; x < 4; ++x) {
              ldsm4t(row + (((x * 2 + (lane >> 4)) ^ (key & 7u)) << 4), vb[x]);
#pragma unroll
              for (uint32_t y = 0; y < 4; ++y) acc |= (vb[x][y] & 0x7FFF7FFFu) + 0x00800080u;
            }
            if (__any_sync(0xFFFFFFFFu, (acc & 0x80008000u) != 0u)) {
              // infinities and NaN among the values: out of the product, and into the rows that see them
#pragma unroll
              for (uint32_t x = 0; x < 4; ++x) {
#pragma unroll
                for (uint32_t y = 0; y < 4; ++y) {
                  const uint32_t bad = ((vb[x][y] & 0x7FFF7FFFu) + 0x00800080u) & 0x80008000u;
                  vb[x][y] &= ~((bad >> 15) * 0xFFFFu);
                }
              }
#pragma unroll 1
              for (uint32_t k = 0; k < 16; ++k) {
                const uint32_t in = g * 16 + k, kr = warp * 32 + in;
                bool see0 = (int32_t)(k0 + in) < hi[0] && ((exist >> in) & 1u), see1 = (int32_t)(k0 + in) < hi[1] && ((exist >> in) & 1u);
                if (MOD && a.m.table) {
                  const int32_t kpos = key_pos(k0 + in);
                  see0 = see0 && __ldg(table[0] + min(max(kpos - qpos[0], -a.m.reach), a.m.reach)) != -INFINITY;
                  see1 = see1 && __ldg(table[1] + min(max(kpos - qpos[1], -a.m.reach), a.m.reach)) != -INFINITY;
                }
                const uint8_t* vrow = gbase + FwSmem::V + s * FW_TILE + kr * 128;
#pragma unroll
                for (uint32_t x = 0; x < 8; ++x) {
                  const uint32_t w2 = *reinterpret_cast<const uint32_t*>(vrow + ((x ^ (kr & 7u)) << 4) + pair * 2);
                  const float v0 = __uint_as_float(w2 << 16), v1 = __uint_as_float(w2 & 0xFFFF0000u);
                  const float a0 = fabsf(v0) < INFINITY ? 0.f : v0, a1 = fabsf(v1) < INFINITY ? 0.f : v1;
                  if (see0) { o[x][0] += a0; o[x][1] += a1; }
                  if (see1) { o[x][2] += a0; o[x][3] += a1; }
                }
              }
            }
#pragma unroll
            for (uint32_t x = 0; x < 4; ++x) {
              mma16816(o[x * 2], pg, vb[x][0], vb[x][1]);
              mma16816(o[x * 2 + 1], pg, vb[x][2], vb[x][3]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(s));
      }
      if (!ok) break;
      // ---- the four warps' parts of the keys, joined
      float* so = reinterpret_cast<float*>(gbase + FwSmem::O);
      float* stat = reinterpret_cast<float*>(gbase + FwSmem::STAT);
#pragma unroll
      for (uint32_t u = 0; u < 2; ++u) {
        l[u] += __shfl_xor_sync(0xFFFFFFFFu, l[u], 1);
        l[u] += __shfl_xor_sync(0xFFFFFFFFu, l[u], 2);
        if ((lane & 3u) == 0) {
          // (a sum that is not a number has no maximum to refer to)
          stat[(warp * 16 + quad + u * 8) * 2] = l[u] != l[u] && m[u] == -INFINITY ? 0.f : m[u];
          stat[(warp * 16 + quad + u * 8) * 2 + 1] = l[u];
        }
      }
      // a row belongs to eight threads (eight columns each); the columns come in two halves
      const uint32_t R = threadIdx.x >> 3, c0 = (threadIdx.x & 7u) * 8;
      float mx = -INFINITY, lt = 0.f, x[8];
#pragma unroll
      for (uint32_t y = 0; y < 8; ++y) x[y] = 0.f;
#pragma unroll
      for (uint32_t half = 0; half < 2; ++half) {
#pragma unroll
        for (uint32_t u = 0; u < 2; ++u) {
#pragma unroll
          for (uint32_t y = 0; y < 4; ++y)
            *reinterpret_cast<float2*>(so + (warp * 16 + quad + u * 8) * 32 + y * 8 + pair) = make_float2(o[half * 4 + y][u * 2], o[half * 4 + y][u * 2 + 1]);
        }
        ok = meet();
        if (!ok) break;
        if (R < rows && (c0 >> 5) == half) {
#pragma unroll
          for (uint32_t w = 0; w < 4; ++w) mx = fmaxf(mx, stat[(w * 16 + R) * 2]);
#pragma unroll
          for (uint32_t w = 0; w < 4; ++w) {
            const float lw = stat[(w * 16 + R) * 2 + 1];
            if (lw == 0.f) continue;                         // nothing seen
            const float f = ex2f(stat[(w * 16 + R) * 2] - mx);
            lt = fmaf(lw, f, lt);
            const float* src = so + (w * 16 + R) * 32 + (c0 & 31u);
#pragma unroll
            for (uint32_t y = 0; y < 8; ++y) x[y] = fmaf(src[y], f, x[y]);
          }
        }
        ok = meet();                                         // (shared memory may be written again)
        if (!ok) break;
      }
      if (!ok) break;
      if (j0 == 0 && j1 == at.nt) {                          // the block has all of it
        if (R < rows) few_output(a, at, R, c0, mx, lt, x);
        continue;
      }
      if (R < rows) {
        // a block has one share that began in it (j0 == 0) and one that began before
        float* slot = p.part + ((size_t)blockIdx.x * 2 + (j0 == 0 ? 1 : 0)) * FW_SLOT;
        float* dst = slot + R * 64 + c0;
        *reinterpret_cast<float4*>(dst) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4*>(dst + 4) = make_float4(x[4], x[5], x[6], x[7]);
        if (c0 == 0) *reinterpret_cast<float2*>(slot + 1024 + R * 2) = make_float2(mx, lt);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(share_out(j0 == 0 ? 1u : 0u));
    }
    if (!ok) { *abort_flag = 1; atomicExch(a.status, 1u); }
  }
  __syncthreads();
}

cudaError_t setup_attn_few() {
  cudaError_t e = cudaFuncSetAttribute(k_attn_few<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, FW_SMEM);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(k_attn_few<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, FW_SMEM);
  return e;
}

size_t attn_few_part_floats(int sm_count) { return (size_t)sm_count * 2 * 2 * FW_SLOT; }

cudaError_t launch_attn_few(const AttnArgs& a, float* part, uint32_t* arrived, int sm_count, cudaStream_t st) {
  alignas(64) CUtensorMap map_k, map_v;
  FwPlan p{};
  const uint32_t ps = 1u << a.page_shift;
  p.page_box = std::min(ps, FW_KEYS);
  p.page_rows = (int)(a.page_stride / 64);
  const uint64_t rows = (uint64_t)(a.num_pages - 1) * (a.page_stride / 64) + (uint64_t)a.kv_heads * ps;
  p.oob_row = (int)rows;
  p.part = part;
  p.arrived = arrived;
  if (!make_tensor_map_bf16(&map_k, a.k_pages, rows, 64, p.page_box) || !make_tensor_map_bf16(&map_v, a.v_pages, rows, 64, p.page_box))
    return cudaErrorInvalidValue;
  // two blocks per SM, but no more than there can be tiles
  const uint64_t cap = std::min<uint64_t>(a.max_len, (uint64_t)a.pages_ld << a.page_shift), tiles = (cap + FW_KEYS - 1) / FW_KEYS;
  const uint64_t grid = std::min<uint64_t>((uint64_t)sm_count * 2, std::max<uint64_t>(1, tiles * a.n_seqs * a.kv_heads));
  const bool mod = a.m.cap > 0.f || a.m.slopes || a.m.table;
  return launch_k(mod ? k_attn_few<true> : k_attn_few<false>, dim3((uint32_t)grid), dim3(FW_THREADS), FW_SMEM, st, map_k, map_v, a, p);
}

}  // namespace llmc
