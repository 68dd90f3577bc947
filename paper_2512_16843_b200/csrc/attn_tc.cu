// Attention on the 5th-generation tensor cores: whole sequences with score modifiers, and chunks over a paged cache.
//
//   S = Q K^T      tcgen05.mma 128 x 128 x 64, operands in shared memory (TMA, 128-byte swizzle), S in tensor memory
//   P = exp2(t - m) t: score in base-2 units with its modifiers; P as bf16 in tensor memory
//   O += P V       tcgen05.mma 128 x 64 x 128, P from tensor memory, V as it lies in memory (MN-major), O in tensor memory
//
// A block works on two tiles of up to 128 query rows that share the key and value tiles.  The query heads that share a
// key/value head are rows of one tile (row = token * group + head of the group), so grouped heads read their keys once and
// few tokens still fill the tile.  Roles: warp 0 walks the block's items (a sequence, a key/value head, 256 rows, and a
// share of the keys where the rows alone do not fill the GPU), decides which key tiles they need and loads them (TMA);
// warps 1 and 2 issue the products of one query tile each; warp 3 looks after what comes with a key tile (document or
// position of every key, missing pages, values that are not numbers); warps 4-7 and 8-11 do the softmax of one query tile
// each, one thread per row: a pass for the maximum (which leaves modified and masked scores in tensor memory) and one for the
// exponentials.  P has columns of its own, so S is free for the next key tile as soon as the second pass has read it, and
// neither product holds up the other.
// What bounds it: the exponentials could be done at 16 per cycle and SM, 1,024 cycles per query and key tile (256 + 256 for
// the two products).  As built a pair of query tiles takes 4,700 cycles per key tile: 870 for the maximum, 2,700 for the
// exponentials (two warps share a scheduler's special function unit, which is busy for 2,050 of them), 500 to 900 until
// the next S is there, the rest barriers.  Measured: 32 prompts of 1,024 tokens, 12 heads, prefix of 512: 144 us (447 TFLOP/s, exponentials
// at 39 % of their rate); 64 rows of 384 tokens in documents: 101 us (1.5 TB/s); 2 rows of 4,001 tokens, 16 heads on 4,
// capped and biased: 195 us; 512 tokens behind 512, 32 sequences, 12 heads: 120 us with the new rows stored; 250 tokens over
// 17,003 and 30,001 keys, 16 heads on 4, capped and biased: 350 us with the weights (123), the join and the new rows.
// Work is handed out by the hardware (cluster launch control): a block for every item is launched, those that run cancel the
// others one by one and do their items.  With item i, i + 148, .. for a block instead the cases took 103, 144, 201, 132 and 389.
// Tried and dropped (the first of these cases, 144 us at the time): maximum and exponentials in one pass over S (160; 384
// instead of 208 with a linear bias, whose growth from key to key makes it start over), S in two halves of 64 keys so that the next one comes
// earlier (153), a quarter of the exponentials by a polynomial on the multiply-add units (148: the time saved goes to the
// wait for S), barriers arrived at by one lane per warp (163), rows kept in registers (195 to 285), two threads per row
// (225), tensor memory read one chunk ahead (155), the two tiles held apart in phase (142).
//
// Maximum: O and the sums refer to a maximum m that is raised, and O scaled, only when a tile's maximum exceeds it by more
// than 2^8: factors up to 2^8 lose nothing in f32 sums and in bf16 P (relative rounding), and O stays in tensor memory.
// Rounding: S, m, sums and O are f32; P is rounded to bf16 (2^-8 relative per weight, averaged over the keys) because the
// product takes bf16 operands; the sums are of the unrounded weights.
//
// Values that are not numbers: P is zero where a key is not seen, but 0 * inf is not.  So infinities and NaN are taken
// out of a V tile before its product (warp 3 scans it: 3 instructions per 4 bytes, hidden behind the exponentials) and
// listed; a row that sees a listed key gets them in its output at the end.
// Every wait is bounded (status word).
#include <cuda.h>
#include <algorithm>
#include "attn_dev.cuh"

namespace llmc {

namespace {

constexpr int TC_THREADS = 384;
constexpr uint32_t TC_ST = 3;                                // stages of the ring of key and value tiles
constexpr uint32_t TC_TILE = 16384;                          // 128 x 64 bf16
constexpr uint32_t TC_KEYS = 128;
constexpr uint32_t TC_TMEM = 512;                            // S0 | S1 (128 columns each) | O0 | O1 | P0 | P1 (64 each)
constexpr uint32_t TC_O = 256, TC_P = 384;
enum : uint32_t { F_NEED0 = 1, F_NEED1 = 2, F_LAST = 4 };            // of a key tile
enum : uint32_t { I_TILES = 1, I_STOP = 2 };                         // of an item: it has key tiles; there are no more items
struct TcSmem {
  static constexpr uint32_t Q = 0;                           // [item parity][query tile]
  static constexpr uint32_t K = Q + 4 * TC_TILE;
  static constexpr uint32_t V = K + TC_ST * TC_TILE;
  static constexpr uint32_t OUT = V + TC_ST * TC_TILE;       // [query tile]: rows on their way out
  static constexpr uint32_t POISON = OUT + 2 * TC_TILE;      // u64 [stage][key][NaN, +inf, -inf]: columns
  static constexpr uint32_t ROWP = POISON + TC_ST * 128 * 24;// u64 [row][3]: the same, seen by a row
  static constexpr uint32_t KINFO = ROWP + 256 * 24;         // i32 [stage][key]: document or position
  static constexpr uint32_t KMASK = KINFO + TC_ST * 512;     // u32 [stage][4]: keys that exist
  static constexpr uint32_t DIRTY = KMASK + TC_ST * 16;      // u32 [stage][4]: keys listed in POISON
  static constexpr uint32_t NRUNS = DIRTY + TC_ST * 16;      // u32 [stage]: runs of keys of one document ...
  static constexpr uint32_t RUNS = NRUNS + 16;               // i32 [stage][128][2]: ... document, first key | end << 16
  static constexpr uint32_t INFO = RUNS + TC_ST * 1024;       // u32 [stage][2]: key tile, flags
  static constexpr uint32_t ITEM = INFO + TC_ST * 8 + 8;         // ItemInfo [2]
  static constexpr uint32_t MAIL = ITEM + 128;               // u32 [query tile][2]: number of the key tile in the block's stream (~0: the item's end), key tile
  static constexpr uint32_t BAR = MAIL + 32;
  static constexpr uint32_t MISC = BAR + 40 * 8;             // [2] words of the block, then the answer to a request for work
  static constexpr uint32_t NEXT = MISC + 32;
  static constexpr uint32_t TOTAL = MISC + 64;
};
static_assert(TcSmem::NEXT % 16 == 0, "an answer of 16 bytes");
constexpr uint32_t TC_SMEM = TcSmem::TOTAL + 1024;
static_assert(TC_SMEM <= 232448, "shared memory of one block");
// kind::f16, f32 accumulator, bf16 operands, M = 128; PV: B is MN-major (bit 16)
constexpr uint32_t TC_IDESC_S = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
constexpr uint32_t TC_IDESC_PV = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((64u >> 3) << 17) | ((128u >> 4) << 24);

// D[tmem] (+)= A[tmem] * B[smem], bf16 inputs, f32 accumulate
__device__ __forceinline__ void tc_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tc_st_16(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
      ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// bits 0 .. n - 1
__device__ __forceinline__ uint32_t below(int32_t n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

// Asks for a block of the grid that has not started: its number arrives at `to` (16 bytes, counted on the barrier).
__device__ __forceinline__ void ask_for_work(uint32_t to, uint32_t bar) {
  mbar_expect_tx(bar, 16);
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(to), "r"(bar) : "memory");
}
// The answer: the block's number, or `none` when all have started (nothing may be asked after that).
__device__ __forceinline__ uint32_t work_answer(uint32_t at, uint32_t none) {
  uint32_t x;
  asm volatile(
      "{\n\t.reg .b128 h;\n\t.reg .pred p;\n\t"
      "ld.shared.b128 h, [%1];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n\t"
      "mov.u32 %0, %2;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, h;\n\t"
      "fence.proxy.async.shared::cta;\n\t}"                 // (the next answer may come to the same place)
      : "=r"(x) : "r"(at), "r"(none) : "memory");
  return x;
}

// Launch shape, the same for every role.
struct TcPlan {
  uint32_t rt;                   // rows of a query tile: the largest multiple of the group up to 128
  uint32_t inv_group;            // ceil(65536 / group): x / group = x * inv_group >> 16 for x < 256
  uint32_t qtiles, splits;       // pairs of query tiles per sequence and head; shares of the keys per item ...
  uint32_t narrow;               // ... and the block's two halves share an item's keys, too (the rows fill one query tile)
  uint32_t shares;               // shares of a row's keys: splits, or twice that
  uint32_t n_items, page_box;    // page_box: rows of a page's box
  int page_rows, oob_row;        // rows of 64 elements between pages; a row behind the last page
  float* part_o;                 // [split][row][head][64], [split][row][head][2] (m, l) when splits > 1
  float* part_ml;
};

struct TcItem {
  uint32_t s, hk, sp, r0, rows;  // rows: those of the sequence (tokens * group)
  SeqGeo g;
  int32_t pre;
  uint32_t ts, te;               // its key tiles ...
  uint32_t mid;                  // ... of which, if narrow, the second half of the block takes those from here on
  bool live;                     // rows of this item exist
};
// keys below this bound may be seen by the row of a token
__device__ __forceinline__ uint32_t keys_to(const AttnArgs& a, uint32_t len, int32_t slot0, int32_t pre, uint32_t token) {
  if (!a.m.causal) return len;
  const int32_t hi = max(slot0 + (int32_t)token + 1, pre);
  return hi <= 0 ? 0u : min((uint32_t)hi, len);
}
__device__ __forceinline__ TcItem tc_item(const AttnArgs& a, const TcPlan& p, uint32_t i, uint32_t n_seqs) {
  TcItem it;
  it.sp = i % p.splits; i /= p.splits;
  it.hk = i % a.kv_heads; i /= a.kv_heads;
  it.s = i % a.n_seqs; i /= a.n_seqs;
  const uint32_t qt = p.qtiles - 1 - i;                      // the tiles with the most keys (causal) first
  it.r0 = qt * 2 * p.rt;
  it.g = SeqGeo{0, a.n, a.n, 0, a.n};
  if (it.s < n_seqs && a.pages) it.g = seq_geo(a, it.s);
  it.pre = a.m.prefix && it.s < n_seqs ? a.m.prefix[it.s] : 0;
  it.rows = it.g.cnt * a.group;
  it.live = it.s < n_seqs && it.r0 < it.rows;
  it.ts = it.te = it.mid = 0;
  if (it.live) {
    const uint32_t nt = (keys_to(a, it.g.len, it.g.slot0, it.pre, (min(it.rows, it.r0 + 2 * p.rt) - 1) / a.group) + TC_KEYS - 1) / TC_KEYS;
    const uint32_t halves = p.narrow ? 2u : 1u, per = (nt + p.shares - 1) / p.shares;
    it.ts = min(nt, it.sp * halves * per);
    it.mid = min(nt, it.ts + per);
    it.te = min(nt, it.ts + halves * per);
  }
  return it;
}
// What the other warps have to know about an item.
struct ItemInfo { uint32_t flags, s, hk, sp, r0, tok0, rows, row0, len; int32_t slot0, pre; };
static_assert(sizeof(ItemInfo) <= 64, "two fit their place in shared memory");
// key tiles that query tile w of an item needs
__device__ __forceinline__ uint32_t tiles_of(const AttnArgs& a, const TcPlan& p, const TcItem& it, uint32_t w) {
  const uint32_t first = it.r0 + w * p.rt;
  if (first >= it.rows) return 0;
  return (keys_to(a, it.g.len, it.g.slot0, it.pre, (min(it.rows, first + p.rt) - 1) / a.group) + TC_KEYS - 1) / TC_KEYS;
}

}  // namespace

// PAGED: keys and values lie in pages; DOC: documents; MOD: scores are capped or biased.  Compiled for each combination that
// a call can have: the roles of a block share an instruction cache that the code of all of them does not fit (with one kernel
// for everything the warps waited for instructions more than for anything else).
template <bool PAGED, bool DOC, bool MOD>
__global__ void __launch_bounds__(TC_THREADS, 1)
k_attn_tc(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
          const __grid_constant__ CUtensorMap map_v, const __grid_constant__ AttnArgs a, const __grid_constant__ TcPlan p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gbase = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t sQ = base + TcSmem::Q, sK = base + TcSmem::K, sV = base + TcSmem::V;
  const uint32_t bar0 = base + TcSmem::BAR;
  auto k_full = [&](uint32_t s) { return bar0 + 8 * s; };
  auto v_full = [&](uint32_t s) { return bar0 + 8 * (TC_ST + s); };
  auto side_full = [&](uint32_t s) { return bar0 + 8 * (2 * TC_ST + s); };
  auto empty = [&](uint32_t s) { return bar0 + 8 * (3 * TC_ST + s); };
  const uint32_t bar1 = bar0 + 8 * 4 * TC_ST;
  auto q_full = [&](uint32_t b) { return bar1 + 8 * b; };
  auto q_empty = [&](uint32_t b) { return bar1 + 8 * (2 + b); };
  auto s_full = [&](uint32_t w) { return bar1 + 8 * (4 + w); };
  auto p_full = [&](uint32_t w) { return bar1 + 8 * (6 + w); };
  auto pv_done = [&](uint32_t w) { return bar1 + 8 * (8 + w); };
  auto s_free = [&](uint32_t w) { return bar1 + 8 * (10 + w); };
  auto drain = [&](uint32_t w) { return bar1 + 8 * (12 + w); };
  const uint32_t asked = bar1 + 8 * 14;
  volatile uint32_t* misc = reinterpret_cast<volatile uint32_t*>(gbase + TcSmem::MISC);
  volatile uint32_t* abort_flag = misc + 1;
  volatile ItemInfo* items = reinterpret_cast<volatile ItemInfo*>(gbase + TcSmem::ITEM);
  volatile uint32_t* info = reinterpret_cast<volatile uint32_t*>(gbase + TcSmem::INFO);
  volatile uint32_t* mail = reinterpret_cast<volatile uint32_t*>(gbase + TcSmem::MAIL);
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < TC_ST; ++s) {
      mbar_init(k_full(s), 1); mbar_init(v_full(s), 1); mbar_init(side_full(s), 1); mbar_init(empty(s), 2 + 8);
    }
    for (uint32_t b = 0; b < 2; ++b) {
      mbar_init(q_full(b), 1); mbar_init(q_empty(b), 2 + 1 + 8); mbar_init(s_full(b), 2); mbar_init(p_full(b), 128);
      mbar_init(pv_done(b), 1); mbar_init(s_free(b), 128); mbar_init(drain(b), 1);
    }
    mbar_init(asked, 1);
    misc[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  // Tensor memory is taken behind the wait for the preceding kernels: a block of theirs on this SM may not have its own yet, and
  // would wait for these columns while this block waits for it.
  griddep_sync();                                            // what the preceding kernels wrote may be read from here on
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32((const void*)misc)), "r"(TC_TMEM) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = misc[0];
  const unsigned long long lim = wait_limit(a.status);
  uint32_t n_seqs = a.n_seqs;
  if (a.n_seqs_dev) n_seqs = min(n_seqs, *a.n_seqs_dev);
  constexpr bool paged = PAGED;

  if (warp < 4) {
  if (warp == 0) {
    // ---------------------------------------------------------------- loads
    bool ok = true;
    // The grid has a block for every item; those that fit the GPU run, and take over the others' items one by one before they
    // start.  The next one is asked for before the work on one begins.
    uint32_t e = 0, qc = 0, n_asked = 0, n_answers = 0;
    const uint32_t sNext = base + TcSmem::NEXT;
    auto next_item = [&]() -> uint32_t {
      ok = warp_wait(asked, (n_asked - 1) & 1u, abort_flag, lim, 64);
      uint32_t x = p.n_items;
      if (ok && lane == 0) x = work_answer(sNext, p.n_items);
      n_answers += ok ? 1u : 0u;
      return __shfl_sync(0xFFFFFFFFu, x, 0);
    };
#pragma unroll 1
    for (uint32_t i = producer_idle(a.status) ? p.n_items : blockIdx.x; i < p.n_items; i = next_item()) {
      if (lane == 0) ask_for_work(sNext, asked);
      ++n_asked;
      const TcItem it = tc_item(a, p, i, n_seqs);
      if (!it.live) continue;
      const uint32_t b = qc & 1u;
      ok = warp_wait(q_empty(b), ((qc >> 1) & 1u) ^ 1u, abort_flag, lim, 64);
      if (!ok) break;
      if (lane == 0) {
        volatile ItemInfo& o = items[b];
        o.flags = it.ts < it.te ? I_TILES : 0u;
        o.s = it.s; o.hk = it.hk; o.sp = it.sp; o.r0 = it.r0; o.tok0 = it.r0 / a.group; o.rows = it.rows; o.row0 = it.g.row0; o.len = it.g.len;
        o.slot0 = it.g.slot0; o.pre = it.pre;
        if (it.ts < it.te) {
          const uint32_t per = p.rt / a.group, bytes = p.rt * 128;
          const int tok = (int)o.tok0 + (paged ? (int)it.g.row0 : 0), seq = paged ? 0 : (int)it.s;
          mbar_expect_tx(q_full(b), 2 * bytes);
          tma_load_4d(sQ + (b * 2) * TC_TILE, &map_q, 0, (int)(it.hk * a.group), tok, seq, q_full(b));
          tma_load_4d(sQ + (b * 2 + 1) * TC_TILE, &map_q, 0, (int)(it.hk * a.group), tok + (p.narrow ? 0 : (int)per), seq, q_full(b));
        } else {
          mbar_arrive(q_full(b));
        }
      }
      ++qc;
      if (it.ts >= it.te) continue;
      const uint32_t nt0 = tiles_of(a, p, it, 0), nt1 = tiles_of(a, p, it, 1);
      const uint32_t n_second = p.narrow ? it.te - it.mid : 0u;
      // smallest and largest document of either query tile (padding left out)
      int32_t lo0 = INT32_MAX, hi0 = -1, lo1 = INT32_MAX, hi1 = -1;
      const int32_t* doc = DOC ? a.m.doc + (size_t)it.s * a.n : nullptr;
      if constexpr (DOC) {
        const uint32_t t0 = it.r0 / a.group, t1 = (it.r0 + p.rt) / a.group, t2 = (it.r0 + 2 * p.rt) / a.group;
#pragma unroll 1
        for (uint32_t t = t0 + lane; t < min(t1, a.n); t += 32) { const int32_t d = doc[t]; if (d >= 0) { lo0 = min(lo0, d); hi0 = max(hi0, d); } }
#pragma unroll 1
        for (uint32_t t = t1 + lane; t < min(t2, a.n); t += 32) { const int32_t d = doc[t]; if (d >= 0) { lo1 = min(lo1, d); hi1 = max(hi1, d); } }
        lo0 = __reduce_min_sync(0xFFFFFFFFu, lo0); hi0 = __reduce_max_sync(0xFFFFFFFFu, hi0);
        lo1 = __reduce_min_sync(0xFFFFFFFFu, lo1); hi1 = __reduce_max_sync(0xFFFFFFFFu, hi1);
      }
      // flags of key tile j (0: nobody needs it)
      auto needs = [&](uint32_t j) -> uint32_t {
        if (PAGED && p.narrow) return j < it.mid ? F_NEED0 : F_NEED1;
        uint32_t f = (j < nt0 ? F_NEED0 : 0u) | (j < nt1 ? F_NEED1 : 0u);
        if (!DOC || !f) return f;
        int32_t lo = INT32_MAX, hi = -1;
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
          const uint32_t k = j * TC_KEYS + u * 32 + lane;
          const int32_t d = k < a.n ? doc[k] : -1;
          if (d >= 0) { lo = min(lo, d); hi = max(hi, d); }
        }
        lo = __reduce_min_sync(0xFFFFFFFFu, lo);
        hi = __reduce_max_sync(0xFFFFFFFFu, hi);
        if (lo > hi0 || hi < lo0) f &= ~F_NEED0;
        if (lo > hi1 || hi < lo1) f &= ~F_NEED1;
        return f;
      };
      // a tile is sent when the next one is known, so that the last one can say so; every item has at least one tile (where
      // documents hide all of them, the last one)
      bool have = false;
      uint32_t j = 0, f = 0;
#pragma unroll 1
      for (uint32_t c = it.ts; c <= it.te; ++c) {
        // (narrow: the halves' tiles in turn, then the rest of the first's)
        uint32_t jc = c;
        if (PAGED && p.narrow) {
          const uint32_t x = c - it.ts;
          jc = x < 2 * n_second ? ((x & 1u) ? it.mid : it.ts) + x / 2 : it.ts + x - n_second;
        }
        uint32_t fc = c < it.te ? needs(jc) : 0u;
        if (!fc && c + 1 == it.te && !have) fc = nt0 > c ? F_NEED0 : F_NEED1;
        if (!fc && c < it.te) continue;
        if (have) {
          if (c == it.te) f |= F_LAST;
          const uint32_t s = e % TC_ST;
          int row = 0;
          const uint32_t boxes = paged ? TC_KEYS / p.page_box : 1u;
          if (paged && lane < boxes) {
            const uint32_t slot = j * TC_KEYS + lane * p.page_box;
            const int32_t pg = slot < it.g.len ? page_of(a, it.s, slot) : -1;
            row = pg < 0 ? p.oob_row
                         : pg * p.page_rows + (int)((it.hk << a.page_shift) + (slot & ((1u << a.page_shift) - 1u)));
          }
          ok = warp_wait(empty(s), ((e / TC_ST) & 1u) ^ 1u, abort_flag, lim, 64);
          if (!ok) break;
          if (lane == 0) {
            info[s * 2] = j;
            info[s * 2 + 1] = f;
            mbar_expect_tx(k_full(s), TC_TILE);
            mbar_expect_tx(v_full(s), TC_TILE);
          }
          __syncwarp();
          if (paged) {
            if (lane < boxes) {
              const uint32_t off = s * TC_TILE + lane * p.page_box * 128;
              tma_load_2d(sK + off, &map_k, 0, row, k_full(s));
              tma_load_2d(sV + off, &map_v, 0, row, v_full(s));
            }
          } else if (lane == 0) {
            tma_load_4d(sK + s * TC_TILE, &map_k, 0, (int)it.hk, (int)(j * TC_KEYS), (int)it.s, k_full(s));
            tma_load_4d(sV + s * TC_TILE, &map_v, 0, (int)it.hk, (int)(j * TC_KEYS), (int)it.s, v_full(s));
          }
          ++e;
        }
        have = true;
        j = jc;
        f = fc;
      }
      if (!ok) break;
    }
    if (ok && !producer_idle(a.status)) {
      ok = warp_wait(q_empty(qc & 1u), ((qc >> 1) & 1u) ^ 1u, abort_flag, lim, 64);
      if (ok && lane == 0) {
        items[qc & 1u].flags = I_STOP;
        mbar_arrive(q_full(qc & 1u));
      }
    }
    if (!ok && lane == 0) { *abort_flag = 1; atomicExch(a.status, 1u); }
    __syncwarp();
    if (lane == 0 && *abort_flag) {
      // a wait ran out: loads in flight must land before the block's shared memory is released
      volatile uint32_t never = 0;
#pragma unroll 1
      for (uint32_t b = 0; b < 2 && b < qc; ++b) wait_long(q_full((qc - 1 - b) & 1u), ((qc - 1 - b) >> 1) & 1u, &never, 200000000ull, 0);
#pragma unroll 1
      for (uint32_t b = 0; b < TC_ST && b < e; ++b) {
        const uint32_t x = e - 1 - b;
        wait_long(k_full(x % TC_ST), (x / TC_ST) & 1u, &never, 200000000ull, 0);
        wait_long(v_full(x % TC_ST), (x / TC_ST) & 1u, &never, 200000000ull, 0);
      }
      // and an answer on its way; the items that nobody has begun are taken and left, so that the grid ends
      bool more = n_asked > n_answers;
#pragma unroll 1
      while (more && wait_long(asked, (n_asked - 1) & 1u, &never, 200000000ull, 0)) {
        more = work_answer(sNext, p.n_items) < p.n_items;
        if (more) { ask_for_work(sNext, asked); ++n_asked; }
      }
    }
  } else if (warp < 3) {
    // ---------------------------------------------------------------- products of query tile w
    // Order: S of a key tile, then P V of the tile before it, so that S is there when its softmax asks for it.
    if (lane == 0) {
      const uint32_t w = warp - 1, need = F_NEED0 << w;
      bool ok = true;
      uint32_t e = 0, n = 0, sent = 0;                       // key tiles of the block; products P V; messages
#pragma unroll 1
      for (uint32_t qc = 0; ok; ++qc) {
        if (!wait_one(q_full(qc & 1u), (qc >> 1) & 1u, abort_flag, lim)) { ok = false; break; }
        const uint32_t flags = items[qc & 1u].flags;
        if (flags & I_STOP) break;
        bool open = false, started = false;                  // a P V is due (of key tile open_e); O has been written
        uint32_t open_e = 0;
        // one turn per key tile and one for the item's end
#pragma unroll 1
        for (bool last = !(flags & I_TILES), end = false; !end;) {
          end = last;
          const uint32_t s = e % TC_ST;
          uint32_t f = 0;
          if (!end) {
            if (!wait_one(k_full(s), (e / TC_ST) & 1u, abort_flag, lim)) { ok = false; break; }
            f = info[s * 2 + 1];
            last = (f & F_LAST) != 0;
          }
          const bool now = (f & need) != 0;
          if (now || end) {
            // a message to the softmax, which has read the one before (and with it the row of S)
            if (sent && !wait_one(s_free(w), (sent - 1) & 1u, abort_flag, lim)) { ok = false; break; }
            ++sent;
            mail[w * 2] = end ? ~0u : e;
            mail[w * 2 + 1] = end ? 0u : info[s * 2];
            if (now) {
              tc_fence_after();
              const uint64_t dq = smem_desc_sw128(sQ + ((qc & 1u) * 2 + w) * TC_TILE), dk = smem_desc_sw128(sK + s * TC_TILE);
#pragma unroll
              for (uint32_t kk = 0; kk < 4; ++kk) tc_mma_bf16(tmem + w * 128, dq + kk * 2, dk + kk * 2, TC_IDESC_S, kk != 0u);
              tc_commit(s_full(w));
            }
            mbar_arrive_n(s_full(w), now ? 1u : 2u);
          }
          if (open) {
            const uint32_t so = open_e % TC_ST;
            if (!wait_one(side_full(so), (open_e / TC_ST) & 1u, abort_flag, lim) ||
                !wait_one(p_full(w), n & 1u, abort_flag, lim)) { ok = false; break; }
            tc_fence_after();
            const uint64_t dv = smem_desc_sw128(sV + so * TC_TILE);
#pragma unroll
            for (uint32_t kk = 0; kk < 8; ++kk)              // 16 keys a step: 2,048 bytes of V, 8 columns of P
              tc_mma_ts(tmem + TC_O + w * 64, tmem + TC_P + w * 64 + kk * 8, dv + kk * 128, TC_IDESC_PV, (started || kk != 0u) ? 1u : 0u);
            tc_commit(pv_done(w));
            tc_commit(empty(so));
            started = true;
            ++n;
          }
          open = now;
          open_e = e;
          if (!end) {
            if (!now) mbar_arrive_n(empty(s), 1 + 4);        // this query tile does not need it, and its softmax does not see it
            ++e;
          }
        }
        if (ok) mbar_arrive(q_empty(qc & 1u));
      }
      if (!ok) {
        *abort_flag = 1;
        atomicExch(a.status, 1u);
        volatile uint32_t never = 0;
        tc_commit(drain(w));                                 // products in flight end before tensor memory is released
        wait_long(drain(w), 0u, &never, 200000000ull, 0);
      }
    }
  } else {
    // ---------------------------------------------------------------- what comes with a key tile
    bool ok = true;
    uint32_t e = 0;
#pragma unroll 1
    for (uint32_t qc = 0; ok; ++qc) {
      ok = warp_wait(q_full(qc & 1u), (qc >> 1) & 1u, abort_flag, lim, 64);
      if (!ok) break;
      volatile ItemInfo& it = items[qc & 1u];
      const uint32_t flags = it.flags, sq = it.s, hk = it.hk, len = it.len;
      if (flags & I_STOP) break;
      const int32_t* src = DOC ? a.m.doc + (size_t)sq * a.n
                           : PAGED && MOD && a.positions ? a.positions + ((size_t)sq * a.kv_heads + hk) * a.side_ld : nullptr;
#pragma unroll 1
      for (bool last = !(flags & I_TILES); !last; ++e) {
        const uint32_t s = e % TC_ST, ph = (e / TC_ST) & 1u;
        ok = warp_wait(k_full(s), ph, abort_flag, lim, 64);
        if (!ok) break;
        const uint32_t j = info[s * 2];
        last = (info[s * 2 + 1] & F_LAST) != 0;
        int32_t* kinfo = reinterpret_cast<int32_t*>(gbase + TcSmem::KINFO) + s * 128;
        uint32_t* kmask = reinterpret_cast<uint32_t*>(gbase + TcSmem::KMASK) + s * 4;
        uint32_t* dirty = reinterpret_cast<uint32_t*>(gbase + TcSmem::DIRTY) + s * 4;
        if ((DOC || (PAGED && MOD)) && src) {
#pragma unroll
          for (uint32_t u = 0; u < 4; ++u) {
            const uint32_t key = j * TC_KEYS + u * 32 + lane;
            kinfo[u * 32 + lane] = key < len ? src[key] : -1;
          }
          if constexpr (DOC) {
            // runs of equal documents: a row's keys are whole runs
            __syncwarp();
            int2* runs = reinterpret_cast<int2*>(gbase + TcSmem::RUNS) + s * 128;
            uint32_t start[4];
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u) {
              const uint32_t c = u * 32 + lane;
              start[u] = __ballot_sync(0xFFFFFFFFu, c == 0 || kinfo[c] != kinfo[c - 1]);
            }
            uint32_t before = 0;
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u) {
              if (start[u] & (1u << lane)) {
                // it ends where the next run starts
                uint32_t end = 128;
                const uint32_t more = start[u] & ~((2u << lane) - 1u);
                if (more) end = u * 32 + __ffs(more) - 1;
                else {
                  for (uint32_t x = u + 1; x < 4; ++x)
                    if (start[x]) { end = x * 32 + __ffs(start[x]) - 1; break; }
                }
                runs[before + __popc(start[u] & ((1u << lane) - 1u))] = make_int2(kinfo[u * 32 + lane], (int)((u * 32 + lane) | (end << 16)));
              }
              before += __popc(start[u]);
            }
            if (lane == 0) reinterpret_cast<uint32_t*>(gbase + TcSmem::NRUNS)[s] = before;
          }
        }
        if (paged) {
#pragma unroll
          for (uint32_t u = 0; u < 4; ++u) {
            const uint32_t key = j * TC_KEYS + u * 32 + lane;
            const uint32_t word = __ballot_sync(0xFFFFFFFFu, key < len && page_of(a, sq, key) >= 0);
            if (lane == 0) kmask[u] = word;
          }
        }
        ok = warp_wait(v_full(s), ph, abort_flag, lim, 64);
        if (!ok) break;
#pragma unroll 1
        for (uint32_t u = 0; u < 4; ++u) {
          const uint32_t c = u * 32 + lane;
          uint8_t* vrow = gbase + TcSmem::V + s * TC_TILE + c * 128;
          // a half with all exponent bits set overflows into its top bit
          uint32_t acc = 0;
#pragma unroll
          for (uint32_t q = 0; q < 8; ++q) {
            const uint4 x = *reinterpret_cast<const uint4*>(vrow + ((q ^ (c & 7u)) << 4));
            acc |= ((x.x & 0x7FFF7FFFu) + 0x00800080u) | ((x.y & 0x7FFF7FFFu) + 0x00800080u) | ((x.z & 0x7FFF7FFFu) + 0x00800080u) |
                   ((x.w & 0x7FFF7FFFu) + 0x00800080u);
          }
          const bool bad = (acc & 0x80008000u) != 0u;
          const uint32_t word = __ballot_sync(0xFFFFFFFFu, bad);
          if (lane == 0) dirty[u] = word;
          if (bad) {
            unsigned long long* ps = reinterpret_cast<unsigned long long*>(gbase + TcSmem::POISON) + (s * 128 + c) * 3;
            unsigned long long nan = 0, pos = 0, neg = 0;
#pragma unroll 1
            for (uint32_t q = 0; q < 8; ++q) {
              uint16_t* h = reinterpret_cast<uint16_t*>(vrow + ((q ^ (c & 7u)) << 4));
#pragma unroll 1
              for (uint32_t x = 0; x < 8; ++x) {
                const uint16_t v = h[x];
                if ((v & 0x7F80u) != 0x7F80u) continue;
                const unsigned long long bit = 1ull << (q * 8 + x);
                if (v & 0x7Fu) nan |= bit; else if (v & 0x8000u) neg |= bit; else pos |= bit;
                h[x] = 0;
              }
            }
            ps[0] = nan; ps[1] = pos; ps[2] = neg;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(side_full(s));
      }
      if (ok && lane == 0) mbar_arrive(q_empty(qc & 1u));
    }
    if (!ok && lane == 0) { *abort_flag = 1; atomicExch(a.status, 1u); }
  }
  } else {
    // ---------------------------------------------------------------- softmax and output, one thread per query row
    const uint32_t w = (warp - 4) >> 2, quarter = warp & 3u, r = quarter * 32 + lane;
    const uint32_t lanes = (quarter * 32u) << 16;
    const uint32_t t_s = tmem + w * 128 + lanes, t_o = tmem + TC_O + w * 64 + lanes, t_p = tmem + TC_P + w * 64 + lanes;
    unsigned long long* rowp = reinterpret_cast<unsigned long long*>(gbase + TcSmem::ROWP) + (w * 128 + r) * 3;
    const float sc = a.m.scale * LOG2E_F;
    constexpr bool side = PAGED || DOC;                      // warp 3's data are needed before the scores are
    // the row's place in its item: an item starts at a multiple of the group
    const uint32_t row0_in = p.narrow ? 0u : w * p.rt, in_item = row0_in + r, my_tok = (in_item * p.inv_group) >> 16, my_head = in_item - my_tok * a.group;
    bool ok = true;
    uint32_t n_msg = 0, n_s = 0;                             // messages; tiles
#pragma unroll 1
    for (uint32_t qc = 0; ok; ++qc) {
      ok = warp_wait(q_full(qc & 1u), (qc >> 1) & 1u, abort_flag, lim, 0);
      if (!ok) break;
      volatile ItemInfo& it = items[qc & 1u];
      if (it.flags & I_STOP) break;
      const uint32_t sq = it.s, hk = it.hk, r0 = it.r0, rows = it.rows, row0 = it.row0, len = it.len, token = it.tok0 + my_tok;
      const int32_t slot0 = it.slot0;
      const uint32_t h = hk * a.group + my_head, left_rows = rows - r0;      // rows of the sequence from the item on
      const bool mine = r < p.rt && in_item < left_rows;     // the row exists
      const int32_t pre = it.pre;
      const uint32_t hi = mine ? keys_to(a, len, slot0, pre, token) : 0u;
      // keys that every row of this tile sees
      const uint32_t all_see = row0_in < left_rows ? keys_to(a, len, slot0, pre, it.tok0 + ((row0_in * p.inv_group) >> 16)) : 0u;
      const int32_t qdoc = DOC && mine ? a.m.doc[(size_t)sq * a.n + token] : -1;
      const int32_t qpos = (PAGED && MOD && a.first ? a.first[sq] : slot0) + (int32_t)token;
      const float slope = MOD && a.m.slopes && mine ? a.m.slopes[h] * LOG2E_F : 0.f;
      const float* table = MOD && a.m.table ? a.m.table + (size_t)(mine ? h : 0u) * (2 * a.m.reach + 1) + a.m.reach : nullptr;
      float m_ref = -INFINITY, l = 0.f;
      bool any = false, poisoned = false;
#pragma unroll 1
      for (;;) {
        ok = warp_wait(s_full(w), n_msg & 1u, abort_flag, lim, 0);
        if (!ok) break;
        ++n_msg;
        const uint32_t e = mail[w * 2], j = mail[w * 2 + 1], s = e % TC_ST;
        if (e == ~0u) {                                      // no more tiles of this item
          mbar_arrive(s_free(w));
          break;
        }
        if (side) {
          ok = warp_wait(side_full(s), (e / TC_ST) & 1u, abort_flag, lim, 0);
          if (!ok) break;
        }
        const int32_t* kinfo = reinterpret_cast<const int32_t*>(gbase + TcSmem::KINFO) + s * 128;
        uint4 km = make_uint4(~0u, ~0u, ~0u, ~0u);
        if (paged) km = *reinterpret_cast<const uint4*>(gbase + TcSmem::KMASK + s * 16);
        // which keys of the tile the row sees, one bit each where it is not all of them
        bool full = (j + 1) * TC_KEYS <= all_see && (km.x & km.y & km.z & km.w) == ~0u;
        uint4 see = km;
        if constexpr (DOC) {
          const int2* runs = reinterpret_cast<const int2*>(gbase + TcSmem::RUNS) + s * 128;
          const uint32_t n_runs = reinterpret_cast<const uint32_t*>(gbase + TcSmem::NRUNS)[s];
          full = full && n_runs == 1 && __all_sync(0xFFFFFFFFu, !mine || (qdoc >= 0 && runs[0].x == qdoc));
          if (!full) {
            see = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 1
            for (uint32_t x = 0; x < n_runs; ++x) {
              const int2 run = runs[x];
              if (run.x == qdoc && qdoc >= 0) {
                const uint32_t first = run.y & 0xFFFFu, end = (uint32_t)run.y >> 16;
                see.x |= below(end) & ~below(first);
                see.y |= below((int)end - 32) & ~below((int)first - 32);
                see.z |= below((int)end - 64) & ~below((int)first - 64);
                see.w |= below((int)end - 96) & ~below((int)first - 96);
              }
            }
          }
        }
        if (!full) {
          const int32_t left = hi > j * TC_KEYS ? (int32_t)min(hi - j * TC_KEYS, TC_KEYS) : 0;
          see.x &= below(left); see.y &= below(left - 32); see.z &= below(left - 64); see.w &= below(left - 96);
        }
        tc_fence_after();
        // distances: the bias is linear over the tile where no seen key lies on the other side of the query, constant where
        // all keys lie beyond the table's reach
        const int32_t d0 = (int32_t)(j * TC_KEYS) - qpos;
        const bool by_key = MOD && PAGED && a.positions && (a.m.slopes || a.m.table);
        const bool linear = MOD && a.m.slopes && !by_key &&
                            __all_sync(0xFFFFFFFFu, (a.m.causal && pre == 0) || d0 >= 0 || d0 + (int32_t)TC_KEYS <= 1);
        // (a causal row's keys beyond the query are masked: their side does not matter)
        const float rise = d0 >= 0 && !(a.m.causal && pre == 0) ? -slope : slope;    // (0 without slopes)
        bool look_up = MOD && a.m.table != nullptr;
        float bias = 0.f;
        if (look_up && !by_key &&
            __all_sync(0xFFFFFFFFu, d0 >= a.m.reach || d0 + (int32_t)TC_KEYS - 1 <= -a.m.reach)) {
          const float b = __ldg(table + (d0 >= a.m.reach ? a.m.reach : -a.m.reach));
          bias = entry2(b);
          look_up = false;
          if (b == -INFINITY) { see = make_uint4(0u, 0u, 0u, 0u); full = false; }
        }
        // whether no score of the tile can go the straight way
        const bool hand = MOD && (by_key || look_up || (a.m.slopes && !linear));
        float mt = -INFINITY;
        if (!MOD && full) {
#pragma unroll 1
          for (uint32_t c = 0; c < 128; c += 32) {
            uint32_t v[32];
            tc_ld_32x32(t_s + c, v);
            tc_wait_ld32(v);
            float m4[4] = {mt, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (uint32_t x = 0; x < 32; x += 8) {
#pragma unroll
              for (uint32_t u = 0; u < 4; ++u) m4[u] = max3f(m4[u], __uint_as_float(v[x + 2 * u]), __uint_as_float(v[x + 2 * u + 1]));
            }
            mt = fmaxf(max3f(m4[0], m4[1], m4[2]), m4[3]);
          }
        } else {
#pragma unroll 1
          for (uint32_t c = 0; c < 128; c += 32) {
            const uint32_t word = c == 0 ? see.x : c == 32 ? see.y : c == 64 ? see.z : see.w;
            uint32_t v[32];
            bool by_hand = hand;
            if (!MOD || !hand) {
            tc_ld_32x32(t_s + c, v);
            tc_wait_ld32(v);
            if constexpr (MOD) {
              const unsigned long long in2 = f2_dup(a.m.cap > 0.f ? a.m.scale / a.m.cap : sc);
              unsigned long long t[16];
#pragma unroll
              for (uint32_t x = 0; x < 16; ++x) t[x] = f2_mul(f2_pack(__uint_as_float(v[2 * x]), __uint_as_float(v[2 * x + 1])), in2);
              if (a.m.cap > 0.f) {
                float big[2] = {0.f, 0.f};
#pragma unroll
                for (uint32_t x = 0; x < 16; ++x) big[x & 1u] = max3f(big[x & 1u], fabsf(f2_lo(t[x])), fabsf(f2_hi(t[x])));
                // (keys that are not seen and rows that do not exist have their say here: it decides how, not what is computed)
                const float most = fmaxf(big[0], big[1]);
                by_hand = by_hand || (mine && !(most <= TANH_TINY));
#pragma unroll
                for (uint32_t x = 0; x < 16; ++x) t[x] = tanh_tiny2(t[x]);
              }
              const unsigned long long u2 = f2_dup(a.m.cap > 0.f ? a.m.cap * LOG2E_F : 1.f), k2 = f2_dup(rise);
              // bias + rise * distance, two keys at a time; each fourth pair anew, so that few roundings add up
              unsigned long long d2 = f2_pack((float)(d0 + (int32_t)c), (float)(d0 + (int32_t)c + 1)), line = 0;
              const unsigned long long b2 = f2_dup(bias), eight = f2_dup(8.f), step = f2_dup(2.f * rise);
#pragma unroll
              for (uint32_t x = 0; x < 16; ++x) {
                if (x % 4 == 0) {
                  line = f2_fma(d2, k2, b2);
                  d2 = f2_add(d2, eight);
                } else {
                  line = f2_add(line, step);
                }
                t[x] = f2_fma(t[x], u2, line);
                v[2 * x] = __float_as_uint(f2_lo(t[x]));
                v[2 * x + 1] = __float_as_uint(f2_hi(t[x]));
              }
            }
            if (!full) {
#pragma unroll
              for (uint32_t x = 0; x < 32; ++x) v[x] = word & (1u << x) ? v[x] : __float_as_uint(-INFINITY);
            }
            }
            if (MOD && __any_sync(0xFFFFFFFFu, by_hand)) {
              // scores beyond the polynomial, distances on both sides, positions, table entries: 16 keys at a time
#pragma unroll 1
              for (uint32_t g = 0; g < 32; g += 16) {
                uint32_t u16[16];
                tc_ld_16(t_s + c + g, u16);
                int32_t d[16];
                float b[16];
#pragma unroll
                for (uint32_t x = 0; x < 16; ++x) d[x] = d0 + (int32_t)(c + g + x);
                if (by_key) {
#pragma unroll
                  for (uint32_t x = 0; x < 16; ++x) d[x] = kinfo[c + g + x] - qpos;
                }
#pragma unroll
                for (uint32_t x = 0; x < 16; ++x) b[x] = 0.f;
                if (look_up) {
#pragma unroll
                  for (uint32_t x = 0; x < 16; ++x) b[x] = __ldg(table + min(max(d[x], -a.m.reach), a.m.reach));
                }
                tc_wait_ld16(u16);
                float z[16];
#pragma unroll
                for (uint32_t x = 0; x < 16; ++x) z[x] = __uint_as_float(u16[x]) * (a.m.cap > 0.f ? a.m.scale / a.m.cap : sc);
                if (a.m.cap > 0.f) {
#pragma unroll
                  for (uint32_t x = 0; x < 16; x += 2) {
                    const unsigned long long t = tanh_any2(f2_pack(z[x], z[x + 1]));
                    z[x] = f2_lo(t) * (hand ? a.m.cap * LOG2E_F : 1.f);
                    z[x + 1] = f2_hi(t) * (hand ? a.m.cap * LOG2E_F : 1.f);
                  }
                }
                if (hand) {
#pragma unroll
                  for (uint32_t x = 0; x < 16; ++x) z[x] = fmaf(-slope, fabsf((float)d[x]), z[x]) + bias + entry2(b[x]);
                } else {
                  // only large scores brought the chunk here: the rest as it is on the straight way, bit for bit
                  const unsigned long long k2 = f2_dup(rise), b2 = f2_dup(bias), eight = f2_dup(8.f), step = f2_dup(2.f * rise);
                  unsigned long long d2 = f2_pack((float)(d0 + (int32_t)c), (float)(d0 + (int32_t)c + 1)), line = 0;
                  if (g) d2 = f2_add(f2_add(d2, eight), eight);
#pragma unroll
                  for (uint32_t x = 0; x < 8; ++x) {
                    if (x % 4 == 0) {
                      line = f2_fma(d2, k2, b2);
                      d2 = f2_add(d2, eight);
                    } else {
                      line = f2_add(line, step);
                    }
                    const unsigned long long t = f2_fma(f2_pack(z[2 * x], z[2 * x + 1]), f2_dup(a.m.cap * LOG2E_F), line);
                    z[2 * x] = f2_lo(t);
                    z[2 * x + 1] = f2_hi(t);
                  }
                }
#pragma unroll
                for (uint32_t x = 0; x < 16; ++x) {
                  z[x] = (word & (1u << (g + x))) && b[x] != -INFINITY ? z[x] : -INFINITY;
                  u16[x] = __float_as_uint(z[x]);
                  mt = fmaxf(mt, z[x]);
                }
                tc_st_16(t_s + c + g, u16);
              }
            } else {
              float m4[4] = {mt, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
              for (uint32_t x = 0; x < 32; x += 8) {
#pragma unroll
                for (uint32_t u = 0; u < 4; ++u) m4[u] = max3f(m4[u], __uint_as_float(v[x + 2 * u]), __uint_as_float(v[x + 2 * u + 1]));
              }
              mt = fmaxf(max3f(m4[0], m4[1], m4[2]), m4[3]);
              tc_st_16(t_s + c, v);                          // for the second pass
              tc_st_16(t_s + c + 16, v + 16);
            }
          }
          tc_wait_st();
        }
        const float unit = MOD ? 1.f : sc;              // base-2 units of what tensor memory holds now
        mt *= unit;
        // P may be written, and O changed, when the product of the tile before has read the one and written the other
        if (any) {
          ok = warp_wait(pv_done(w), (n_s - 1) & 1u, abort_flag, lim, 0);
          if (!ok) break;
          tc_fence_after();
        }
        ++n_s;
        // raise the reference maximum?
        const bool raise = mt > m_ref + 8.f;
        if (!any) {
          m_ref = mt;
          any = true;
        } else if (__any_sync(0xFFFFFFFFu, raise)) {
          const float m_new = raise ? mt : m_ref;
          const float corr = raise ? ex2f(m_ref - m_new) : 1.f;
          l *= corr;
          m_ref = m_new;
          const unsigned long long c2 = f2_dup(corr);
#pragma unroll 1
          for (uint32_t c = 0; c < 64; c += 16) {
            uint32_t o[16];
            tc_ld_16(t_o + c, o);
            tc_wait_ld16(o);
#pragma unroll
            for (uint32_t x = 0; x < 8; ++x) {
              const unsigned long long y = f2_mul(f2_pack(__uint_as_float(o[2 * x]), __uint_as_float(o[2 * x + 1])), c2);
              o[2 * x] = __float_as_uint(f2_lo(y));
              o[2 * x + 1] = __float_as_uint(f2_hi(y));
            }
            tc_st_16(t_o + c, o);
          }
        }
        const unsigned long long nm2 = f2_dup(m_ref == -INFINITY ? 0.f : -m_ref), sc2 = f2_dup(unit);
        float l0 = 0.f, l1 = 0.f;
#pragma unroll 1
        for (uint32_t c = 0; c < 128; c += 32) {
          uint32_t v[32], pk[16];
          tc_ld_32x32(t_s + c, v);
          tc_wait_ld32(v);
          if (c == 96) {                                     // the row is read: the next key tile's S may come
            tc_fence_before();
            mbar_arrive(s_free(w));
          }
#pragma unroll
          for (uint32_t x = 0; x < 16; ++x) {
            const unsigned long long t2 = f2_fma(f2_pack(__uint_as_float(v[2 * x]), __uint_as_float(v[2 * x + 1])), sc2, nm2);
            const float pa = ex2f(f2_lo(t2)), pb = ex2f(f2_hi(t2));
            l0 += pa;
            l1 += pb;
            pk[x] = pack2(pa, pb);
          }
          tc_st_16(t_p + c / 2, pk);
        }
        l += l0 + l1;
        tc_wait_st();
        tc_fence_before();
        mbar_arrive(p_full(w));
        if (!side) {
          ok = warp_wait(side_full(s), (e / TC_ST) & 1u, abort_flag, lim, 0);
          if (!ok) break;
        }
        const uint4 dw = *reinterpret_cast<const uint4*>(gbase + TcSmem::DIRTY + s * 16);
        if (dw.x | dw.y | dw.z | dw.w) {
          // values that are not numbers: note the columns in which this row sees them
          const uint32_t listed[4] = {full ? dw.x : dw.x & see.x, full ? dw.y : dw.y & see.y, full ? dw.z : dw.z & see.z, full ? dw.w : dw.w & see.w};
#pragma unroll 1
          for (uint32_t c = 0; c < 128; ++c) {
            const uint32_t word = c < 32 ? listed[0] : c < 64 ? listed[1] : c < 96 ? listed[2] : listed[3];
            if (!((word >> (c & 31u)) & 1u)) continue;
            if (MOD && look_up) {
              const int32_t d = by_key ? kinfo[c] - qpos : d0 + (int32_t)c;
              if (__ldg(table + min(max(d, -a.m.reach), a.m.reach)) == -INFINITY) continue;
            }
            const unsigned long long* ps = reinterpret_cast<const unsigned long long*>(gbase + TcSmem::POISON) + (s * 128 + c) * 3;
#pragma unroll 1
            for (uint32_t x = 0; x < 3; ++x) rowp[x] = (poisoned ? rowp[x] : 0ull) | ps[x];
            poisoned = true;
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(s));
      }
      if (!ok) break;
      // ---- output
      const bool dead = l == 0.f;                            // nothing seen
      const float inv = dead ? 0.f : 1.f / l;
      if (any) {
        ok = warp_wait(pv_done(w), (n_s - 1) & 1u, abort_flag, lim, 0);
        if (!ok) break;
        tc_fence_after();
      }
      const uint32_t sp = p.narrow ? it.sp * 2 + w : it.sp;
      const size_t n_rowids = (size_t)a.n_rows * a.heads;    // of a paged call
      const size_t rowid = (paged ? (size_t)row0 + token : (size_t)sq * a.n + token) * a.heads + h;
      const uint32_t tok0 = it.tok0;
      __syncwarp();
      if (lane == 0) mbar_arrive(q_empty(qc & 1u));          // the item's description has been read
      // rows of 128 bytes go through shared memory, so that eight lanes store one (each warp its own 32 rows)
      uint8_t* stage = gbase + TcSmem::OUT + w * TC_TILE + quarter * 32 * 128;
      float* part = p.part_o + ((size_t)sp * n_rowids + rowid) * 64;
#pragma unroll 1
      for (uint32_t c = 0; c < 64; c += 16) {
        uint32_t v[16];
        if (any) {
          tc_ld_16(t_o + c, v);
          tc_wait_ld16(v);
        }
#pragma unroll
        for (uint32_t x = 0; x < 16; ++x) v[x] = dead ? 0u : v[x];
        if (p.shares > 1) {
          if (mine) {
#pragma unroll
            for (uint32_t x = 0; x < 16; x += 4)
              *reinterpret_cast<uint4*>(part + c + x) = make_uint4(v[x], v[x + 1], v[x + 2], v[x + 3]);
          }
        } else {
#pragma unroll
          for (uint32_t x = 0; x < 8; ++x) v[x] = pack2(__uint_as_float(v[2 * x]) * inv, __uint_as_float(v[2 * x + 1]) * inv);
          *reinterpret_cast<uint4*>(stage + lane * 128 + (((c >> 3) ^ (lane & 7u)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
          *reinterpret_cast<uint4*>(stage + lane * 128 + (((c >> 3) + 1 ^ (lane & 7u)) << 4)) = make_uint4(v[4], v[5], v[6], v[7]);
        }
        __syncwarp();
      }
      if (poisoned && !dead && mine) {
        // columns in which the row saw values that are not numbers (a row whose sum is NaN keeps it)
#pragma unroll 1
        for (unsigned long long bits = rowp[0] | rowp[1] | rowp[2]; bits; bits &= bits - 1) {
          const uint32_t c = __ffsll((long long)bits) - 1;
          const bool nan = ((rowp[0] | (rowp[1] & rowp[2])) >> c) & 1ull || l != l, neg = (rowp[2] >> c) & 1ull;
          const float x = nan ? NAN : neg ? -INFINITY : INFINITY;
          if (p.shares > 1) part[c] = x;
          else *reinterpret_cast<__nv_bfloat16*>(stage + lane * 128 + (((c >> 3) ^ (lane & 7u)) << 4) + (c & 7u) * 2) = __float2bfloat16_rn(x);
        }
      }
      __syncwarp();
      if (mine) {
        if (p.shares > 1)
          reinterpret_cast<float2*>(p.part_ml)[(size_t)sp * n_rowids + rowid] = make_float2(l != l && m_ref == -INFINITY ? 0.f : m_ref, l);
        else {
          if (a.lse) a.lse[rowid] = dead ? -INFINITY : log_sum(m_ref, l);
          if (a.stat) a.stat[rowid] = make_float2(m_ref, l);
        }
      }
      if (p.shares == 1) {
        __nv_bfloat16* out0 = a.out.ptr + (paged ? (long long)row0 * a.out.tok : (long long)sq * a.out.seq) + (long long)tok0 * a.out.tok +
                              (long long)hk * a.group * a.out.head + (lane & 7u) * 8;
#pragma unroll 1
        for (uint32_t rr = lane >> 3; rr < 32; rr += 4) {
          const uint32_t in_tile = quarter * 32 + rr, ii = row0_in + in_tile, tk = (ii * p.inv_group) >> 16;
          if (in_tile < p.rt && ii < left_rows)
            *reinterpret_cast<uint4*>(out0 + (long long)tk * a.out.tok + (long long)(ii - tk * a.group) * a.out.head) =
                *reinterpret_cast<const uint4*>(stage + rr * 128 + (((lane & 7u) ^ (rr & 7u)) << 4));
        }
      }
      __syncwarp();                                          // (the next item's rows come to the same place)
    }
    if (!ok) { *abort_flag = 1; atomicExch(a.status, 1u); }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TC_TMEM) : "memory");
  }
}

// The shares of the keys of one row joined: one warp per row and head of a paged call, two columns per lane.
__global__ void __launch_bounds__(256) k_attn_join(const AttnArgs a, const float* part_o, const float* part_ml, uint32_t splits) {
  griddep_sync();
  const uint32_t lane = threadIdx.x & 31;
  const size_t n_rowids = (size_t)a.n_rows * a.heads;
  for (size_t id = ((size_t)blockIdx.x * 256 + threadIdx.x) >> 5; id < n_rowids; id += (size_t)gridDim.x * 8) {
    const uint32_t row = (uint32_t)(id / a.heads), h = (uint32_t)(id % a.heads);
    const SeqGeo g = seq_geo(a, seq_of_row(a, row));
    if (row < g.row0 || row - g.row0 >= g.cnt) continue;     // belongs to no sequence of the call
    // a lane looks after every 32nd share: the maximum first, then the factors, which all lanes need
    const float2* ml = reinterpret_cast<const float2*>(part_ml) + id;
    float m = -INFINITY;
    for (uint32_t s = lane; s < splits; s += 32) m = fmaxf(m, ml[(size_t)s * n_rowids].x);
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    float l = 0.f;
    float2 o = make_float2(0.f, 0.f);
    if (m != -INFINITY) {
      for (uint32_t s0 = 0; s0 < splits; s0 += 32) {
        float2 mine = make_float2(0.f, 0.f);
        if (s0 + lane < splits) mine = ml[(size_t)(s0 + lane) * n_rowids];
        const float c = mine.y == 0.f ? 0.f : ex2f(mine.x - m);      // nothing seen in this share: it takes no part
        const uint32_t n = min(32u, splits - s0);
#pragma unroll 4
        for (uint32_t u = 0; u < n; ++u) {
          const float2 x = *reinterpret_cast<const float2*>(part_o + ((size_t)(s0 + u) * n_rowids + id) * 64 + lane * 2);
          const float f = __shfl_sync(0xFFFFFFFFu, c, u), y = __shfl_sync(0xFFFFFFFFu, mine.y, u);
          if (y == 0.f) continue;
          l = fmaf(y, f, l);
          o.x = fmaf(x.x, f, o.x);
          o.y = fmaf(x.y, f, o.y);
        }
      }
    }
    const float inv = m == -INFINITY ? 0.f : 1.f / l;
    *reinterpret_cast<uint32_t*>(a.out.ptr + (long long)row * a.out.tok + (long long)h * a.out.head + lane * 2) = pack2(o.x * inv, o.y * inv);
    if (a.lse && lane == 0) a.lse[id] = m == -INFINITY ? -INFINITY : log_sum(m, l);
    if (a.stat && lane == 0) a.stat[id] = make_float2(m, l);
  }
}

namespace {
using TcKernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const AttnArgs, const TcPlan);
TcKernel tc_kernel(bool paged, bool doc, bool mod) {
  if (paged) return mod ? k_attn_tc<true, false, true> : k_attn_tc<true, false, false>;
  if (doc) return mod ? k_attn_tc<false, true, true> : k_attn_tc<false, true, false>;
  return mod ? k_attn_tc<false, false, true> : k_attn_tc<false, false, false>;
}
}  // namespace

cudaError_t setup_attn_tc() {
  cudaError_t e = tensor_map_setup();
  for (int i = 0; i < 6 && e == cudaSuccess; ++i)
    e = cudaFuncSetAttribute(tc_kernel(i / 2 == 2, i / 2 == 1, i & 1), cudaFuncAttributeMaxDynamicSharedMemorySize, TC_SMEM);
  return e;
}

// A call over whole sequences, or over a paged cache.  part: scratch for part_units x (row, head, share) results of a
// paged call (66 floats each), or null: the keys are not split.
cudaError_t launch_attn_tc(const AttnArgs& a, float* part, size_t part_units, int sm_count, cudaStream_t st) {
  if (a.n_seqs == 0 || a.n == 0) return cudaSuccess;
  const bool paged = a.pages != nullptr;
  alignas(64) CUtensorMap map_q, map_k, map_v;
  TcPlan p{};
  p.rt = 128 / a.group * a.group;
  p.inv_group = (65536 + a.group - 1) / a.group;
  const uint64_t seq_rows = (uint64_t)a.n * a.group;
  p.qtiles = (uint32_t)((seq_rows + 2 * p.rt - 1) / (2 * p.rt));
  p.splits = 1;
  const uint64_t items = (uint64_t)p.qtiles * a.n_seqs * a.kv_heads;
  p.shares = 1;
  if (paged && part) {
    const uint64_t cap = std::min<uint64_t>(a.max_len, (uint64_t)a.pages_ld << a.page_shift), tiles = (cap + TC_KEYS - 1) / TC_KEYS;
    const uint64_t rows = (uint64_t)a.n_rows * a.heads;
    // rows that fill one query tile: both halves of a block work on them, with the keys shared out between them.  33 rows, 12
    // heads, 64 sequences, without and with: capped and biased over 640 keys 124 and 114 us, over 2,560 404 and 312; positions and a
    // table over 640 200 and 171; plain over 640 79 and 81, over 2,600 298 and 279.  Few items pay for it (4 sequences, 640
    // keys: capped and biased 27 and 32, plain 24 and 26), and below four key tiles nobody gains (300 keys: 116 and 128)
    p.narrow = seq_rows <= p.rt && tiles >= 4 && part_units / rows >= 2;
    const uint64_t halves = p.narrow ? 2 : 1;
    // as many shares as it takes to give every SM an item (of two key tiles at least), and up to three items per SM where they
    // stay long (16 tiles), because sequences of uneven lengths then end together.  One, two, three items per SM: 250 rows over
    // 17,003 and 30,001 keys, capped and biased, 288, 245, 246 us (230 with four, for which the scratch has no room); 200 rows over
    // 3,000 to 30,000 keys 148, 124, 116; 100 over 4,000 to 16,000 146, 151, 134; even lengths pay for it: 250 rows over twice
    // 24,000 keys 117, 114, 128, 512 over 30,000 110, 118, 140
    uint64_t sp = std::min<uint64_t>((uint64_t)sm_count / items, (tiles + 1) / 2 / halves);
    sp = std::max<uint64_t>(sp, std::min<uint64_t>(3ull * sm_count / items, tiles / 16 / halves));
    sp = std::min<uint64_t>(sp, part_units / rows / halves);
    if (sp > 1) p.splits = (uint32_t)sp;
    p.shares = p.splits * (uint32_t)halves;
    p.part_o = part;
    p.part_ml = part + (size_t)p.shares * rows * 64;
  }
  if (items * p.splits > 0x7FFFFFFFull) return cudaErrorInvalidValue;
  p.n_items = (uint32_t)(items * p.splits);
  const uint64_t seqs = paged ? 1 : a.n_seqs, toks = paged ? a.n_rows : a.n;
  if (!make_tensor_map_rows(&map_q, a.q, a.heads, toks, seqs, a.group, p.rt / a.group)) return cudaErrorInvalidValue;
  if (paged) {
    const uint32_t ps = 1u << a.page_shift;
    p.page_box = ps < TC_KEYS ? ps : TC_KEYS;
    p.page_rows = (int)(a.page_stride / 64);
    const uint64_t rows = (uint64_t)(a.num_pages - 1) * (a.page_stride / 64) + (uint64_t)a.kv_heads * ps;
    p.oob_row = (int)rows;
    if (!make_tensor_map_bf16(&map_k, a.k_pages, rows, 64, p.page_box) || !make_tensor_map_bf16(&map_v, a.v_pages, rows, 64, p.page_box))
      return cudaErrorInvalidValue;
  } else {
    if (!make_tensor_map_rows(&map_k, a.k, a.kv_heads, a.n, a.n_seqs, 1, TC_KEYS) ||
        !make_tensor_map_rows(&map_v, a.v, a.kv_heads, a.n, a.n_seqs, 1, TC_KEYS))
      return cudaErrorInvalidValue;
  }
  const bool mod = a.m.cap > 0.f || a.m.slopes || a.m.table;
  cudaError_t e = launch_k(tc_kernel(paged, a.m.doc != nullptr, mod), dim3(p.n_items), dim3(TC_THREADS), TC_SMEM, st, map_q, map_k, map_v, a, p);
  if (e != cudaSuccess || p.shares == 1) return e;
  const uint64_t warps = (uint64_t)a.n_rows * a.heads;
  const uint64_t blocks = std::min<uint64_t>((warps + 7) / 8, (uint64_t)sm_count * 8);
  return launch_k(k_attn_join, dim3((uint32_t)blocks), dim3(256), 0, st, a, (const float*)p.part_o, (const float*)p.part_ml, p.shares);
}

}  // namespace llmc
