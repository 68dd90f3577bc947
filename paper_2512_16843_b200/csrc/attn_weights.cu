// Received weights of a paged call: weights[key] = decay * weights[key] + sum over the call's rows, and over the query heads
// that share the key, of exp(z - m) / l (m, l: maximum and sum of the row, as the attention left them).  The scores are formed again, with the keys as the rows of the product:
//   S^T = K Q^T    tcgen05.mma 128 keys x up to 128 query rows x 64
// so that a thread owns a key and its sum over the rows needs no exchange and no atomics (same bits every time).  What a
// row adds to a score is prepared once per tile: -(m + log l), and with a linear bias slope * (first key - query) with the slope
// beside it, so that a score costs one or two multiply-adds and its exponential.  A block
// takes a sequence and head and every parts-th key tile of it; the query rows stream past each key tile (they come from
// L2).  Two groups of four warps take turns with the query tiles, two blocks per SM.  Reads K once more (128 bytes per
// key and head) and the queries; one exponential per score, as in the attention itself.
// Measured: 250 tokens over 17,003 and 30,001 keys, 16 heads on 4, capped and biased: 123 us (147 million scores; the
// schedulers issue in 64 % of their cycles, the capped score's multiply-adds above all).
// f32 throughout; every wait is bounded (status word).
#include <algorithm>
#include "attn_dev.cuh"

namespace llmc {

namespace {

constexpr int WT_THREADS = 384;                              // warp 0: loads, 1: products, 2-3: row data, 4-11: sums
constexpr uint32_t WT_ST = 3, WT_TILE = 16384, WT_KEYS = 128, WT_TMEM = 256;
struct WtSmem {
  static constexpr uint32_t K = 0;                           // [2]
  static constexpr uint32_t Q = K + 2 * WT_TILE;             // [WT_ST]
  static constexpr uint32_t ADD = Q + WT_ST * WT_TILE;       // f32 [stage][128], base 2: - (m + log l) (- inf: the row gives nothing) + linear bias
  static constexpr uint32_t TOP = ADD + WT_ST * 512;         // f32 [stage][128][2]: - m and 1 / l (where scores are large, log l is lost beside m)
  static constexpr uint32_t SLOPE = TOP + WT_ST * 1024;      // f32 [stage][128]
  static constexpr uint32_t QPOS = SLOPE + WT_ST * 512;      // i32 [stage][128]
  static constexpr uint32_t HI = QPOS + WT_ST * 512;         // i32 [stage][128]: keys below it are seen
  static constexpr uint32_t TAB = HI + WT_ST * 512;          // i32 [stage][128]: middle of the head's row of the table
  static constexpr uint32_t XCH = TAB + WT_ST * 512;         // f32 [2][128]
  static constexpr uint32_t BAR = XCH + 1024;
  static constexpr uint32_t MISC = BAR + 24 * 8;
  static constexpr uint32_t TOTAL = MISC + 64;
};
constexpr uint32_t WT_SMEM = WtSmem::TOTAL + 1024;

struct WtPlan {
  uint32_t rt, cols;             // query rows per tile; columns of the product (rt rounded up to 16)
  uint32_t parts, page_box;
  int page_rows, oob_row;
};

}  // namespace

// MOD: scores are capped or biased.
template <bool MOD>
__global__ void __launch_bounds__(WT_THREADS, 2)
k_attn_weights(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
               const __grid_constant__ AttnArgs a, const __grid_constant__ WtPlan p) {
  griddep_sync();
  const uint32_t part = blockIdx.x % p.parts, hk = (blockIdx.x / p.parts) % a.kv_heads, sq = blockIdx.x / p.parts / a.kv_heads;
  const SeqGeo g = seq_geo(a, sq);
  const uint32_t rows = g.cnt * a.group, nt = (g.len + WT_KEYS - 1) / WT_KEYS, qtiles = (rows + p.rt - 1) / p.rt;
  if (part >= nt) return;                                    // uniform over the block; nothing allocated yet
  const size_t side0 = ((size_t)sq * a.kv_heads + hk) * a.side_ld;
  if (rows == 0) {                                           // no rows: what was received before fades
    for (uint32_t j = part; j < nt; j += p.parts)
      for (uint32_t c = threadIdx.x; c < WT_KEYS; c += WT_THREADS)
        if (j * WT_KEYS + c < g.len) {
          float& w = a.weights[side0 + j * WT_KEYS + c];
          w = a.decay == 0.f ? 0.f : a.decay * w;
        }
    return;
  }
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gbase = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bar0 = base + WtSmem::BAR;
  auto q_full = [&](uint32_t s) { return bar0 + 8 * s; };
  auto side_full = [&](uint32_t s) { return bar0 + 8 * (WT_ST + s); };
  auto empty = [&](uint32_t s) { return bar0 + 8 * (2 * WT_ST + s); };
  const uint32_t bar1 = bar0 + 8 * 3 * WT_ST;
  auto k_full = [&](uint32_t b) { return bar1 + 8 * b; };
  auto k_empty = [&](uint32_t b) { return bar1 + 8 * (2 + b); };
  auto s_full = [&](uint32_t w) { return bar1 + 8 * (4 + w); };
  auto s_empty = [&](uint32_t w) { return bar1 + 8 * (6 + w); };
  auto x_full = [&](uint32_t b) { return bar1 + 8 * (8 + b); };
  auto x_empty = [&](uint32_t b) { return bar1 + 8 * (10 + b); };
  const uint32_t drain = bar1 + 8 * 12;
  volatile uint32_t* misc = reinterpret_cast<volatile uint32_t*>(gbase + WtSmem::MISC);
  volatile uint32_t* abort_flag = misc + 1;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned long long lim = wait_limit(a.status);
  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < WT_ST; ++s) { mbar_init(q_full(s), 1); mbar_init(side_full(s), 2); mbar_init(empty(s), 1 + 4); }
    for (uint32_t b = 0; b < 2; ++b) {
      mbar_init(k_full(b), 1); mbar_init(k_empty(b), 1); mbar_init(s_full(b), 1); mbar_init(s_empty(b), 128);
      mbar_init(x_full(b), 128); mbar_init(x_empty(b), 128);
    }
    mbar_init(drain, 1);
    misc[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32((const void*)misc)), "r"(WT_TMEM) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = misc[0];

  // entry n of the block: key tile number n / qtiles of its own, query tile n % qtiles; group n % 2 of the summing warps
  if (warp == 0) {
    bool ok = true;
    uint32_t n = 0, t = 0;
    for (uint32_t j = producer_idle(a.status) ? nt : part; j < nt && ok; j += p.parts, ++t) {
      const uint32_t boxes = WT_KEYS / p.page_box;
      int row = 0;
      if (lane < boxes) {
        const uint32_t slot = j * WT_KEYS + lane * p.page_box;
        const int32_t pg = slot < g.len ? page_of(a, sq, slot) : -1;
        row = pg < 0 ? p.oob_row : pg * p.page_rows + (int)((hk << a.page_shift) + (slot & ((1u << a.page_shift) - 1u)));
      }
      ok = warp_wait(k_empty(t & 1u), ((t >> 1) & 1u) ^ 1u, abort_flag, lim, 32);
      if (!ok) break;
      if (lane == 0) mbar_expect_tx(k_full(t & 1u), WT_TILE);
      __syncwarp();
      if (lane < boxes) tma_load_2d(base + WtSmem::K + (t & 1u) * WT_TILE + lane * p.page_box * 128, &map_k, 0, row, k_full(t & 1u));
      for (uint32_t qt = 0; qt < qtiles; ++qt, ++n) {
        const uint32_t s = n % WT_ST;
        ok = warp_wait(empty(s), ((n / WT_ST) & 1u) ^ 1u, abort_flag, lim, 32);
        if (!ok) break;
        if (lane == 0) {
          mbar_expect_tx(q_full(s), p.rt * 128);
          tma_load_4d(base + WtSmem::Q + s * WT_TILE, &map_q, 0, (int)(hk * a.group), (int)(g.row0 + qt * (p.rt / a.group)), 0, q_full(s));
        }
      }
    }
    if (!ok && lane == 0) { *abort_flag = 1; atomicExch(a.status, 1u); }
    __syncwarp();
    if (lane == 0 && *abort_flag) {                          // loads in flight must land before shared memory is released
      volatile uint32_t never = 0;
      const uint32_t tk = ok ? t : t + 1;
      for (uint32_t b = 0; b < 2 && b < tk; ++b) mbar_wait(k_full((tk - 1 - b) & 1u), ((tk - 1 - b) >> 1) & 1u, &never, 200000000ull);
      for (uint32_t b = 0; b < WT_ST && b < n; ++b) mbar_wait(q_full((n - 1 - b) % WT_ST), ((n - 1 - b) / WT_ST) & 1u, &never, 200000000ull);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((p.cols >> 3) << 17) | ((128u >> 4) << 24);
      bool ok = true;
      uint32_t n = 0, t = 0;
      for (uint32_t j = part; j < nt && ok; j += p.parts, ++t) {
        if (!mbar_wait(k_full(t & 1u), (t >> 1) & 1u, abort_flag, lim, 32)) { ok = false; break; }
        const uint64_t dk = smem_desc_sw128(base + WtSmem::K + (t & 1u) * WT_TILE);
        for (uint32_t qt = 0; qt < qtiles; ++qt, ++n) {
          const uint32_t s = n % WT_ST, w = n & 1u;
          if (!mbar_wait(q_full(s), (n / WT_ST) & 1u, abort_flag, lim, 32) ||
              !mbar_wait(s_empty(w), ((n >> 1) & 1u) ^ 1u, abort_flag, lim, 20)) { ok = false; break; }
          tc_fence_after();
          const uint64_t dq = smem_desc_sw128(base + WtSmem::Q + s * WT_TILE);
#pragma unroll
          for (uint32_t kk = 0; kk < 4; ++kk) tc_mma_bf16(tmem + w * 128, dk + kk * 2, dq + kk * 2, idesc, kk != 0u);
          tc_commit(s_full(w));
          tc_commit(empty(s));
        }
        if (ok) tc_commit(k_empty(t & 1u));
      }
      if (!ok) {
        *abort_flag = 1;
        atomicExch(a.status, 1u);
        volatile uint32_t never = 0;
        tc_commit(drain);
        mbar_wait(drain, 0u, &never, 200000000ull);
      }
    }
  } else if (warp < 4) {
    bool ok = true;
    const int32_t pos0 = a.first ? a.first[sq] : g.slot0;
    const uint32_t total = ((nt - part + p.parts - 1) / p.parts) * qtiles;
    for (uint32_t n = 0; n < total; ++n) {
      const uint32_t s = n % WT_ST, qt = n % qtiles, j = part + n / qtiles * p.parts;
      ok = warp_wait(empty(s), ((n / WT_ST) & 1u) ^ 1u, abort_flag, lim, 32);
      if (!ok) break;
#pragma unroll 1
      for (uint32_t u = 0; u < 2; ++u) {
        const uint32_t c = u * 64 + threadIdx.x - 64, R = qt * p.rt + c;
        const uint32_t token = R / a.group, h = hk * a.group + R % a.group;
        const bool real = c < p.rt && R < rows;
        float2 ml = make_float2(0.f, 0.f);
        if (real) ml = a.stat[(size_t)(g.row0 + token) * a.heads + h];
        const bool none = ml.y == 0.f;                       // a row that sees nothing gives nothing
        const float add = none ? -INFINITY : -(ml.x + lg2f(ml.y));
        const uint32_t at = s * 128 + c;
        const int32_t qpos = pos0 + (int32_t)token;
        const float slope = MOD && a.m.slopes && real ? a.m.slopes[h] * LOG2E_F : 0.f;
        reinterpret_cast<float*>(gbase + WtSmem::ADD)[at] = fmaf(slope, (float)((int32_t)(j * WT_KEYS) - qpos), add);
        reinterpret_cast<int32_t*>(gbase + WtSmem::HI)[at] =
            !real ? 0 : a.m.causal ? min(g.slot0 + (int32_t)token + 1, (int32_t)g.len) : (int32_t)g.len;
        if constexpr (MOD) {
          reinterpret_cast<float2*>(gbase + WtSmem::TOP)[at] = none ? make_float2(0.f, 0.f) : make_float2(-ml.x, 1.f / ml.y);
          reinterpret_cast<float*>(gbase + WtSmem::SLOPE)[at] = slope;
          reinterpret_cast<int32_t*>(gbase + WtSmem::QPOS)[at] = qpos;
          if (a.m.table) reinterpret_cast<int32_t*>(gbase + WtSmem::TAB)[at] = (int32_t)((real ? h : 0u) * (2 * a.m.reach + 1)) + a.m.reach;
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(side_full(s));
    }
    if (!ok && lane == 0) { *abort_flag = 1; atomicExch(a.status, 1u); }
  } else {
    const uint32_t w = (warp - 4) >> 2, quarter = warp & 3u, key_in = quarter * 32 + lane;
    const uint32_t t_s = tmem + w * 128 + ((quarter * 32u) << 16);
    const float unit = a.m.cap > 0.f ? a.m.cap * LOG2E_F : a.m.scale * LOG2E_F;
    // the straight path needs keys that lie before their queries, at their slots
    const bool odd = MOD && (a.m.table || (a.m.slopes && (a.positions || !a.m.causal)));
    float* xch = reinterpret_cast<float*>(gbase + WtSmem::XCH);
    bool ok = true;
    uint32_t n = 0, mine = 0, t = 0;                         // entries of the block, of this group; key tiles
    for (uint32_t j = part; j < nt && ok; j += p.parts, ++t) {
      const uint32_t key = j * WT_KEYS + key_in;
      const bool real = key < g.len;
      const bool there = real && page_of(a, sq, key) >= 0;
      const int32_t kpos = a.positions && real ? a.positions[side0 + key] : (int32_t)key;
      float sum = 0.f;
      for (uint32_t qt = 0; qt < qtiles; ++qt, ++n) {
        if ((n & 1u) != w) continue;
        const uint32_t s = n % WT_ST;
        ok = warp_wait(side_full(s), (n / WT_ST) & 1u, abort_flag, lim, 32) && warp_wait(s_full(w), mine & 1u, abort_flag, lim, 20);
        if (!ok) break;
        ++mine;
        tc_fence_after();
        const float* add = reinterpret_cast<const float*>(gbase + WtSmem::ADD) + s * 128;
        const float* slope = reinterpret_cast<const float*>(gbase + WtSmem::SLOPE) + s * 128;
        const int32_t* hi = reinterpret_cast<const int32_t*>(gbase + WtSmem::HI) + s * 128;
        const uint32_t n_rows = min(p.rt, rows - qt * p.rt);
        float s0 = 0.f, s1 = 0.f;
#pragma unroll 1
        for (uint32_t c = 0; c < n_rows; c += 32) {
          uint32_t v[32];
          tc_ld_32x32(t_s + c, v);
          // (the rows of a tile see ever more keys: the first row of the chunk sees the fewest)
          const bool all = c + 32 <= n_rows && hi[c] >= (int32_t)((j + 1) * WT_KEYS);
          bool by_hand = odd;
          tc_wait_ld32(v);
          if constexpr (MOD) {
            if (a.m.cap > 0.f) {
              const unsigned long long in2 = f2_dup(a.m.scale / a.m.cap);
              float big[2] = {0.f, 0.f};
              unsigned long long t[16];
              const uint32_t left = n_rows - c;
#pragma unroll
              for (uint32_t i = 0; i < 16; ++i) {
                t[i] = f2_mul(f2_pack(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), in2);
                // (columns behind the last row hold whatever was there before)
                big[i & 1u] = max3f(big[i & 1u], 2 * i < left ? fabsf(f2_lo(t[i])) : 0.f, 2 * i + 1 < left ? fabsf(f2_hi(t[i])) : 0.f);
              }
              const float most = fmaxf(big[0], big[1]);
              by_hand = by_hand || (real && !(most <= TANH_TINY));
#pragma unroll
              for (uint32_t i = 0; i < 16; ++i) t[i] = tanh_tiny2(t[i]);
#pragma unroll
              for (uint32_t i = 0; i < 16; ++i) {
                v[2 * i] = __float_as_uint(f2_lo(t[i]));
                v[2 * i + 1] = __float_as_uint(f2_hi(t[i]));
              }
            }
          }
          if (!MOD || !__any_sync(0xFFFFFFFFu, by_hand)) {
            const unsigned long long u2 = f2_dup(unit), k2 = f2_dup((float)key_in);
#pragma unroll
            for (uint32_t i = 0; i < 32; i += 4) {
              const float4 b = *reinterpret_cast<const float4*>(add + c + i);
              unsigned long long x0 = f2_fma(f2_pack(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), u2, f2_pack(b.x, b.y));
              unsigned long long x1 = f2_fma(f2_pack(__uint_as_float(v[i + 2]), __uint_as_float(v[i + 3])), u2, f2_pack(b.z, b.w));
              if (MOD) {
                const float4 sl = *reinterpret_cast<const float4*>(slope + c + i);
                x0 = f2_fma(f2_pack(sl.x, sl.y), k2, x0);
                x1 = f2_fma(f2_pack(sl.z, sl.w), k2, x1);
              }
              float p0 = ex2f(f2_lo(x0)), p1 = ex2f(f2_hi(x0)), p2 = ex2f(f2_lo(x1)), p3 = ex2f(f2_hi(x1));
              if (!all) {
                const int4 q = *reinterpret_cast<const int4*>(hi + c + i);
                p0 = (int32_t)key < q.x ? p0 : 0.f;
                p1 = (int32_t)key < q.y ? p1 : 0.f;
                p2 = (int32_t)key < q.z ? p2 : 0.f;
                p3 = (int32_t)key < q.w ? p3 : 0.f;
              }
              s0 += p0 + p2;
              s1 += p1 + p3;
            }
          } else {
            // scores beyond the polynomial, positions, distances on both sides, table entries: 16 rows at a time
            const float2* top = reinterpret_cast<const float2*>(gbase + WtSmem::TOP) + s * 128;
            const int32_t* qpos = reinterpret_cast<const int32_t*>(gbase + WtSmem::QPOS) + s * 128;
            const int32_t* tab = reinterpret_cast<const int32_t*>(gbase + WtSmem::TAB) + s * 128;
#pragma unroll 1
            for (uint32_t o = c; o < min(c + 32, n_rows); o += 16) {
              uint32_t u[16];
              tc_ld_16(t_s + o, u);
              float b[16], z[16];
#pragma unroll
              for (uint32_t i = 0; i < 16; ++i) b[i] = 0.f;
              if (a.m.table) {
#pragma unroll
                for (uint32_t i = 0; i < 16; ++i)
                  b[i] = o + i < n_rows ? __ldg(a.m.table + tab[o + i] + min(max(kpos - qpos[o + i], -a.m.reach), a.m.reach)) : 0.f;
              }
              tc_wait_ld16(u);
#pragma unroll
              for (uint32_t i = 0; i < 16; ++i) z[i] = __uint_as_float(u[i]) * (a.m.cap > 0.f ? a.m.scale / a.m.cap : unit);
              if (a.m.cap > 0.f) {
#pragma unroll
                for (uint32_t i = 0; i < 16; i += 2) {
                  const unsigned long long t = tanh_any2(f2_pack(z[i], z[i + 1]));
                  z[i] = f2_lo(t) * (odd ? unit : 1.f);
                  z[i + 1] = f2_hi(t) * (odd ? unit : 1.f);
                }
              }
              if (!odd) {
                // only large scores brought the chunk here: the rest as it is on the straight way, bit for bit
#pragma unroll
                for (uint32_t i = 0; i < 16; ++i) {
                  z[i] = ex2f(fmaf(slope[o + i], (float)key_in, fmaf(z[i], unit, add[o + i])));
                  z[i] = (int32_t)key < hi[o + i] ? z[i] : 0.f;
                }
#pragma unroll
                for (uint32_t i = 0; i < 16; i += 4) {
                  s0 += z[i] + z[i + 2];
                  s1 += z[i + 1] + z[i + 3];
                }
                continue;
              }
#pragma unroll
              for (uint32_t i = 0; i < 16; ++i) {
                z[i] = fmaf(-slope[o + i], fabsf((float)(kpos - qpos[o + i])), z[i]) + entry2(b[i]) + top[o + i].x;
                const float x = ex2f(z[i]) * top[o + i].y;
                s0 += (int32_t)key < hi[o + i] && b[i] != -INFINITY ? x : 0.f;
              }
            }
          }
        }
        sum += s0 + s1;
        tc_fence_before();
        mbar_arrive(s_empty(w));
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(s));
      }
      if (!ok) break;
      // several query tiles: the two groups' sums are added; one: the group that had it stores
      bool store = real && ((n - 1) & 1u) == w;
      if (qtiles > 1) {
        float* x = xch + (t & 1u) * 128;
        const uint32_t ph = (t >> 1) & 1u;
        if (w == 1) {
          ok = warp_wait(x_empty(t & 1u), ph ^ 1u, abort_flag, lim, 20);
          if (!ok) break;
          x[key_in] = sum;
          mbar_arrive(x_full(t & 1u));
        } else {
          ok = warp_wait(x_full(t & 1u), ph, abort_flag, lim, 20);
          if (!ok) break;
          sum += x[key_in];
          mbar_arrive(x_empty(t & 1u));
        }
        store = real && w == 0;
      }
      if (store) {
        float& dst = a.weights[side0 + key];
        const float got = there ? sum : 0.f;
        dst = a.decay == 0.f ? got : fmaf(a.decay, dst, got);
      }
    }
    if (!ok) { *abort_flag = 1; atomicExch(a.status, 1u); }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(WT_TMEM) : "memory");
  }
}

cudaError_t setup_attn_kernels() {
  cudaError_t e = setup_attn_tc();
  if (e == cudaSuccess) e = setup_attn_few();
  if (e == cudaSuccess) e = cudaFuncSetAttribute(k_attn_weights<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, WT_SMEM);
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(k_attn_weights<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, WT_SMEM);
}

bool attn_is_few(const AttnArgs& a) {
  if (!a.pages || (uint64_t)a.n * a.group > FEW_ROWS) return false;
  const uint64_t cap = std::min<uint64_t>(a.max_len, (uint64_t)a.pages_ld << a.page_shift);
  return (cap / 128 + 1) * a.n_seqs * a.kv_heads < (1ull << 31);          // (its tiles are counted in 32 bits)
}

cudaError_t launch_attn(const AttnArgs& a, const AttnScratch& s, int sm_count, cudaStream_t st) {
  if (attn_is_few(a)) return launch_attn_few(a, s.part, s.arrived, sm_count, st);
  return launch_attn_tc(a, s.part, s.part_units, sm_count, st);
}

// The weights of a call whose scores k_attn_few left: one thread per key, blocks in turn over the keys of a sequence and
// head.  Reads 4 bytes per row and key, once (they are still in L2 as a rule).  9 us for 64
// sequences of 301 to 4,100 slots, 16 heads on 4; forming those scores again took 36.
__global__ void __launch_bounds__(256) k_weights_of_scores(const __grid_constant__ AttnArgs a, uint32_t parts) {
  griddep_sync();
  const uint32_t part = blockIdx.x % parts, hk = (blockIdx.x / parts) % a.kv_heads, sq = blockIdx.x / parts / a.kv_heads;
  const SeqGeo g = seq_geo(a, sq);
  const uint32_t rows = g.cnt * a.group;
  __shared__ float top[FEW_ROWS], inv[FEW_ROWS];
  if (threadIdx.x < rows) {
    const float2 ml = a.stat[(size_t)(g.row0 + threadIdx.x / a.group) * a.heads + hk * a.group + threadIdx.x % a.group];
    const bool none = ml.y == 0.f;                           // a row that sees nothing gives nothing
    top[threadIdx.x] = none ? 0.f : ml.x;
    inv[threadIdx.x] = none ? 0.f : 1.f / ml.y;
  }
  __syncthreads();
  const size_t pair = (size_t)sq * a.kv_heads + hk;
  const float* scores = a.scores + pair * a.score_rows * a.score_ld;
  for (uint32_t key = part * 256 + threadIdx.x; key < g.len; key += parts * 256) {
    float sum = 0.f;
#pragma unroll 4
    for (uint32_t R = 0; R < rows; ++R) sum = fmaf(ex2f(__ldcg(scores + (size_t)R * a.score_ld + key) - top[R]), inv[R], sum);
    float& w = a.weights[pair * a.side_ld + key];
    w = a.decay == 0.f ? sum : fmaf(a.decay, w, sum);
  }
}

cudaError_t launch_attn_weights(const AttnArgs& a, int sm_count, cudaStream_t st) {
  if (a.n_seqs == 0) return cudaSuccess;
  if (a.scores) {
    const uint64_t pairs = (uint64_t)a.n_seqs * a.kv_heads, chunks = (a.score_ld + 255) / 256;
    const uint32_t parts = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(chunks, ((uint64_t)sm_count * 8 + pairs - 1) / pairs));
    if (pairs * parts > 0x7FFFFFFFull) return cudaErrorInvalidValue;
    return launch_k(k_weights_of_scores, dim3((uint32_t)(pairs * parts)), dim3(256), 0, st, a, parts);
  }
  alignas(64) CUtensorMap map_q, map_k;
  WtPlan p{};
  const uint32_t toks = std::min(128 / a.group, a.n);        // tokens of a query tile
  p.rt = toks * a.group;
  p.cols = (p.rt + 15) / 16 * 16;
  const uint32_t ps = 1u << a.page_shift;
  p.page_box = std::min(ps, WT_KEYS);
  p.page_rows = (int)(a.page_stride / 64);
  const uint64_t rows = (uint64_t)(a.num_pages - 1) * (a.page_stride / 64) + (uint64_t)a.kv_heads * ps;
  p.oob_row = (int)rows;
  const uint64_t cap = std::min<uint64_t>(a.max_len, (uint64_t)a.pages_ld << a.page_shift), tiles = (cap + WT_KEYS - 1) / WT_KEYS;
  // about eight blocks per SM: enough for even shares, few enough that the ends of wide tables cost little
  const uint64_t pairs = (uint64_t)a.n_seqs * a.kv_heads, want = ((uint64_t)sm_count * 8 + pairs - 1) / pairs;
  p.parts = (uint32_t)std::min(tiles, want);
  if (pairs * p.parts > 0x7FFFFFFFull) return cudaErrorInvalidValue;
  if (!make_tensor_map_rows(&map_q, a.q, a.heads, a.n_rows, 1, a.group, toks) ||
      !make_tensor_map_bf16(&map_k, a.k_pages, rows, 64, p.page_box))
    return cudaErrorInvalidValue;
  const bool mod = a.m.cap > 0.f || a.m.slopes || a.m.table;
  return launch_k(mod ? k_attn_weights<true> : k_attn_weights<false>, dim3((uint32_t)(pairs * p.parts)), dim3(WT_THREADS), WT_SMEM, st, map_q, map_k, a, p);
}

}  // namespace llmc
