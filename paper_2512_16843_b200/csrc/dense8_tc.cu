// Product of two 8-bit matrices on the tensor cores:
//   out[m, n] = act(a_scale[m] w_scale[n] sum_k a[m, k] w[n, k] + bias[n]) (+ residual[m, n]),   bf16 out
// int8 is summed in 32-bit integers (exact: k <= 131,056), e4m3 in fp32.
//
// Tiles of 128 bytes of k come by TMA (128-byte swizzle, zeros beyond the matrices' ends) into a ring; tcgen05.mma sums them in one
// of two accumulators in tensor memory while the epilogue drains the other.  Large products take a pair of blocks per 256 x 256
// tile (cta_group::2): each block loads its 128 rows of a and 128 of w and keeps 128 rows of the accumulator, so a block's copies are
// 64 bytes per cycle at the tensor cores' full rate where a tile of its own would need 96.  Small ones take 128 x 128 or 128 x 64 per
// block, or clusters that share their k (dense8_split.cu), by estimated time (below).  One elected lane of a warp issues copies, products and
// commits: behind a branch on lane 0 the compiler issues each in a loop over lanes, and a step of k of a block alone took 275 ns whatever its tile.  A step of
// one tile alone, rows on 128 bytes, takes 157 ns for 128 x 128 (239 with rows on 32 bytes, 360 on 16), 192 for 128 x 64 (192, 270) and 262 to 292
// for a pair's (the same, 360); with all SMs at work 195 to 225, 200 to 220 and 290 to 370.
// 32,768 x 4,096 x 1,024 112 us, 120 to 127 with GELU (2,450 and 2,230 T operations per second); 65,536 x 1,024 x 4,096 179, e4m3 with residual 197 to 209;
// 1,001 x 50,257 x 768 43 to 48.
//
// An epilogue warp has 32 rows x 64 columns of its own and a box of 4 KB in shared memory for them: the residual comes into
// the box by TMA while the tile is still being summed, the result takes its place and leaves by TMA in rows of 128 bytes.  Warps meet
// nowhere but at the accumulator's barriers; scales and biases are read through L1, the same address in all lanes.  Four warps for each 64
// columns: the steps of one (tensor memory, arithmetic, box, copy) are a chain that only other warps can cover.
// The number of valid rows may come from device memory.  All mbarrier waits are bounded (status word).
#include <cuda.h>
#include "dense8.cuh"
#include "layer_epi.cuh"

namespace llmc {

namespace {
constexpr int DM = 128, DK = 128;                   // rows of a block's accumulator; bytes of k per step
constexpr uint32_t DA_BYTES = DM * DK;
constexpr uint32_t D_BOX = 32 * 128;                // a warp's 32 rows of 64 columns

// CTAS blocks share a tile of CTAS * 128 rows and BN columns
template <int CTAS, int BN>
struct D8 {
  static constexpr int STAGES = CTAS == 2 ? 5 : BN == 128 ? 6 : 8;
  static constexpr int EPI_WARPS = 4 * (BN / 64);
  static constexpr int THREADS = 64 + 32 * EPI_WARPS;             // warp 0: TMA, warp 1: MMA, then the epilogue
  static constexpr uint32_t B_BYTES = BN / CTAS * DK;
  static constexpr uint32_t A = 0;
  static constexpr uint32_t B = A + STAGES * DA_BYTES;
  static constexpr uint32_t BOX = B + STAGES * B_BYTES;           // one per epilogue warp
  static constexpr uint32_t BAR = BOX + EPI_WARPS * D_BOX;
  static constexpr uint32_t MISC = BAR + (2 * STAGES + 4 + EPI_WARPS) * 8;
  static constexpr uint32_t BYTES = MISC + 16 + 1024;
  static constexpr uint32_t TMEM = 2 * BN;
  static_assert(BYTES <= 232448, "shared memory of one block");
};

__device__ __forceinline__ float4 ldg4(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }

__device__ __align__(16) const float d8_no_bias[64] = {};

// 16 columns of a row: scales s, biases b, activation, residual r (pairs of bf16); y: pairs of neighbouring columns
template <bool I8, uint32_t ACT, bool RES>
__device__ __forceinline__ void finish16(const uint32_t (&v)[16], unsigned long long sa2, const float (&s)[16], const float (&b)[16],
                                         const uint32_t (&r)[8], unsigned long long (&y)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const unsigned long long x = I8 ? f2_pack((float)(int32_t)v[2 * j], (float)(int32_t)v[2 * j + 1])
                                    : f2_pack(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
    y[j] = f2_fma(f2_mul(x, sa2), f2_pack(s[2 * j], s[2 * j + 1]), f2_pack(b[2 * j], b[2 * j + 1]));
  }
  if (ACT != LAYER_ACT_NONE) {
    gelu_phi2_x8<ACT == LAYER_ACT_GELU_TANH, RES>(y, r);
  } else if (RES) {
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = f2_add(y[j], bf16_pair(r[j]));
  }
}
__device__ __forceinline__ void put4(uint4 v, uint32_t* r) { r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w; }
__device__ __forceinline__ uint4 bf16x8(const unsigned long long* y) {
  return make_uint4(pack_bf16(f2_lo(y[0]), f2_hi(y[0])), pack_bf16(f2_lo(y[1]), f2_hi(y[1])), pack_bf16(f2_lo(y[2]), f2_hi(y[2])),
                    pack_bf16(f2_lo(y[3]), f2_hi(y[3])));
}
// A warp's 32 rows of 64 columns from its box to memory by plain copies, two columns per lane, eight rows at a time: rows and columns beyond the
// ends stay out.
__device__ __noinline__ void plain_box(__nv_bfloat16* at, long long ld, uint32_t row0, uint32_t col0, uint32_t M, uint32_t N, uint32_t box, uint32_t lane) {
  const uint32_t col = col0 + 2 * lane, rows = min(32u, M - row0);
#pragma unroll 1
  for (uint32_t r0 = 0; r0 < rows; r0 += 8) {
    uint32_t w[8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[i]) : "r"(box + (r0 + i) * 128 + (((lane >> 2) ^ i) << 4) + (lane & 3u) * 4) : "memory");
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      __nv_bfloat16* p = at + (long long)(row0 + r0 + i) * ld + col;
      if (r0 + i >= rows) break;
      if (col + 1 < N) *reinterpret_cast<uint32_t*>(p) = w[i];
      else if (col < N) *p = __ushort_as_bfloat16((unsigned short)w[i]);
    }
  }
  __syncwarp();
}
}  // namespace

// I8: int8 or e4m3; ACT, RES, VT as in the bf16 product: each epilogue carries only its own code
template <int CTAS, int BN, bool I8, uint32_t ACT, bool RES, bool VT>
__global__ void __launch_bounds__((D8<CTAS, BN>::THREADS), 1)
k_dense8_tc(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_w,
            const __grid_constant__ CUtensorMap map_out, const __grid_constant__ CUtensorMap map_res, const DenseArgs p) {
  griddep_sync();
  using S = D8<CTAS, BN>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;           // (the same in both blocks of a pair)
  uint8_t* gbase = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t sA = base + S::A, sB = base + S::B, bar0 = base + S::BAR;
  auto full_bar = [&](uint32_t s) { return bar0 + 8 * s; };                              // pair: rank 0's counts both blocks' copies
  auto empty_bar = [&](uint32_t s) { return bar0 + 8 * (S::STAGES + s); };
  auto tfull_bar = [&](uint32_t b) { return bar0 + 8 * (2 * S::STAGES + b); };
  auto tempty_bar = [&](uint32_t b) { return bar0 + 8 * (2 * S::STAGES + 2 + b); };      // pair: rank 0's counts both blocks' warps
  auto res_bar = [&](uint32_t w) { return bar0 + 8 * (2 * S::STAGES + 4 + w); };         // one per epilogue warp
  volatile uint32_t* misc = reinterpret_cast<volatile uint32_t*>(gbase + S::MISC);
  volatile uint32_t* tmem_slot = misc + 0;
  volatile uint32_t* abort_flag = misc + 1;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CTAS == 2 ? pair_rank() : 0u;
  const unsigned long long lim = wait_limit(p.status);

  const uint32_t M = rows_of(p.m, p.count_dev, p.rows_per_count), N = p.n;
  const uint32_t KB = (p.k + DK - 1) / DK;
  const uint32_t MB = (M + CTAS * DM - 1) / (CTAS * DM), NB = (N + BN - 1) / BN;
  const uint32_t n_tiles = MB * NB, first = blockIdx.x / CTAS, step = gridDim.x / CTAS;
  // neighbouring blocks work on neighbours along the shorter side, so that what they read at a time is small
  auto tile_mb = [&](uint32_t t) { return MB <= NB ? t % MB : t / NB; };
  auto tile_nb = [&](uint32_t t) { return MB <= NB ? t / MB : t % NB; };

  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < (uint32_t)S::STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (uint32_t b = 0; b < 2; ++b) {
      mbar_init(tfull_bar(b), 1);
      mbar_init(tempty_bar(b), CTAS * S::EPI_WARPS);
    }
    for (uint32_t w = 0; w < (uint32_t)S::EPI_WARPS; ++w) mbar_init(res_bar(w), 1);
    misc[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    if constexpr (CTAS == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                   ::"r"(smem_u32((const void*)tmem_slot)), "r"(S::TMEM) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                   ::"r"(smem_u32((const void*)tmem_slot)), "r"(S::TMEM) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  __syncwarp();
  if constexpr (CTAS == 2) pair_meet();            // the other block's barriers are ready too
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  uint32_t issued = 0;
  const bool leader = elect_one();
  if (warp == 0) {
    if (leader && !producer_idle(p.status)) {       // ---- TMA producer
      bool ok = true;
      for (uint32_t t = first; t < n_tiles && ok; t += step) {
        const int row = (int)(tile_mb(t) * (CTAS * DM) + rank * DM), col = (int)(tile_nb(t) * BN + rank * (BN / CTAS));
        for (uint32_t kb = 0; kb < KB; ++kb) {
          const uint32_t s = issued % S::STAGES, ph = (issued / S::STAGES) & 1u;
          if (!mbar_wait(empty_bar(s), ph ^ 1u, abort_flag, lim)) { ok = false; break; }
          if (rank == 0) mbar_expect_tx(full_bar(s), CTAS * (DA_BYTES + S::B_BYTES));
          if constexpr (CTAS == 2) {
            const uint32_t bar = of_rank0(full_bar(s));
            tma_load_2d_pair(sA + s * DA_BYTES, &map_a, (int)(kb * DK), row, bar);
            tma_load_2d_pair(sB + s * S::B_BYTES, &map_w, (int)(kb * DK), col, bar);
          } else {
            tma_load_2d(sA + s * DA_BYTES, &map_a, (int)(kb * DK), row, full_bar(s));
            tma_load_2d(sB + s * S::B_BYTES, &map_w, (int)(kb * DK), col, full_bar(s));
          }
          ++issued;
        }
      }
      // pair: what the other block's products signal here must have arrived before the block ends
      for (uint32_t i = 0; CTAS == 2 && ok && i < (uint32_t)S::STAGES && i < issued; ++i) {
        const uint32_t x = issued - 1 - i;
        ok = mbar_wait(empty_bar(x % S::STAGES), (x / S::STAGES) & 1u, abort_flag, lim);
      }
      if (!ok) { *abort_flag = 1; atomicExch(p.status, 1u); }
    }
  } else if (warp == 1) {
    if (leader && rank == 0) {                         // ---- MMA issuer
      // operand types: signed 8-bit integers into 32-bit ones, or e4m3 into fp32
      constexpr uint32_t idesc = (I8 ? (2u << 4) | (1u << 7) | (1u << 10) : (1u << 4)) | ((uint32_t)(BN >> 3) << 17) |
                                 ((uint32_t)((CTAS * DM) >> 4) << 24);
      bool ok = true;
      uint32_t it = 0, tile = 0;
      for (uint32_t t = first; t < n_tiles && ok; t += step, ++tile) {
        const uint32_t buf = tile & 1u, bph = (tile >> 1) & 1u;
        if (!mbar_wait(tempty_bar(buf), bph ^ 1u, abort_flag, lim)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + buf * BN;
        for (uint32_t kb = 0; kb < KB; ++kb, ++it) {
          const uint32_t s = it % S::STAGES, ph = (it / S::STAGES) & 1u;
          if (!mbar_wait(full_bar(s), ph, abort_flag, lim)) { ok = false; break; }
          tc_fence_after();
          const uint64_t da = smem_desc_sw128(sA + s * DA_BYTES), db = smem_desc_sw128(sB + s * S::B_BYTES);
#pragma unroll
          for (uint32_t kk = 0; kk < DK / 32; ++kk) {
            const uint32_t more = (kb | kk) != 0u;
            if constexpr (CTAS == 2) {
              if (I8) tc_mma_i8_pair(d_tmem, da + kk * 2, db + kk * 2, idesc, more);
              else    tc_mma_f8_pair(d_tmem, da + kk * 2, db + kk * 2, idesc, more);
            } else {
              if (I8) tc_mma_i8(d_tmem, da + kk * 2, db + kk * 2, idesc, more);
              else    tc_mma_f8(d_tmem, da + kk * 2, db + kk * 2, idesc, more);
            }
          }
          if constexpr (CTAS == 2) tc_commit_pair(empty_bar(s)); else tc_commit(empty_bar(s));
        }
        if (ok) { if constexpr (CTAS == 2) tc_commit_pair(tfull_bar(buf)); else tc_commit(tfull_bar(buf)); }
      }
      if (!ok) { *abort_flag = 1; atomicExch(p.status, 1u); }
    }
  } else {
    // ---- epilogue: a lane = one row of the tile, 64 columns of it
    const uint32_t ew = warp - 2, quarter = warp & 3u, col_in_tile = (ew >> 2) * 64;
    const uint32_t row_in_tile = rank * DM + quarter * 32;
    const uint32_t box = base + S::BOX + ew * D_BOX;
    const uint32_t my_row = (box + lane * 128u) | ((lane & 7u) << 4);      // piece c of the row is at my_row ^ (c << 4): the swizzle
    // The copy engine cuts columns off in pieces of 16 bytes, so that it stores up to N8 and the lanes the rest, each of its row.  Plain
    // stores for the rows of a partial block whose number came from the device.
    const uint32_t N8 = N & ~7u;
    uint32_t r_issued = 0, r_used = 0;
    auto fetch_residual = [&](uint32_t t) {            // (the leader; the box is free.  Rows from M to p.m are there too)
      if (t >= n_tiles) return;
      const uint32_t row0 = tile_mb(t) * (CTAS * DM) + row_in_tile, col0 = tile_nb(t) * BN + col_in_tile;
      if (row0 >= M || col0 >= N) return;
      mbar_expect_tx(res_bar(ew), D_BOX);
      tma_load_2d(box, &map_res, (int)col0, (int)row0, res_bar(ew));
      ++r_issued;
    };
    if (RES && leader) fetch_residual(first);
    uint32_t tile = 0;
    bool live = true;
    for (uint32_t t = first; t < n_tiles && live; t += step, ++tile) {
      const uint32_t buf = tile & 1u, bph = (tile >> 1) & 1u;
      const uint32_t row0 = tile_mb(t) * (CTAS * DM) + row_in_tile, col0 = tile_nb(t) * BN + col_in_tile;
      const uint32_t row = row0 + lane;
      const bool some = row0 < M && col0 < N, whole_rows = M == p.m || row0 + 32 <= M;
      const float sa = row < M ? __ldg(p.a_scale + row) : 0.f;
      // a wait that ran out ends the warp's work: nothing more is read, and nothing asked for that is not waited for
      live = __all_sync(0xFFFFFFFFu, mbar_wait(tfull_bar(buf), bph, abort_flag, lim));
      if (live && RES && some) {
        live = __all_sync(0xFFFFFFFFu, mbar_wait(res_bar(ew), r_used & 1u, abort_flag, lim));
        if (live) ++r_used;
      }
      if (!live) { *abort_flag = 1; atomicExch(p.status, 1u); break; }
      tc_fence_after();
      const uint32_t taddr = tmem_base + buf * BN + col_in_tile + ((quarter * 32u) << 16);
      const unsigned long long sa2 = f2_pack(sa, sa);
      const bool transposed = VT && col0 >= p.vt.col0;
      const float* ws = p.w_scale + col0;
      const float* bs = p.bias ? p.bias + col0 : d8_no_bias;
      auto release = [&]() {                           // the accumulator's columns are in registers: it may be filled again
        tc_fence_before();
        __syncwarp();
        if (leader) {
          if constexpr (CTAS == 2) mbar_arrive_cluster(of_rank0(tempty_bar(buf))); else mbar_arrive(tempty_bar(buf));
        }
      };
      auto sixteen = [&](uint32_t u, const uint32_t (&v)[16], const float (&s)[16], const float (&b)[16]) {
        uint32_t r[8];
        unsigned long long y[8];
        if (RES) {
          put4(lds16(my_row ^ ((u * 2) << 4)), r);
          put4(lds16(my_row ^ ((u * 2 + 1) << 4)), r + 4);
        }
        finish16<I8, ACT, RES>(v, sa2, s, b, r, y);
        if (!transposed) {
          sts16(my_row ^ ((u * 2) << 4), bf16x8(y));
          sts16(my_row ^ ((u * 2 + 1) << 4), bf16x8(y + 4));
        } else if (row < M) {
          // the V third of a q|k|v product, transposed per head (see the bf16 product); lanes are neighbouring positions
          const uint32_t seq = row / p.rows_per_count, pos = row - seq * p.rows_per_count;
          __nv_bfloat16* dst = p.vt.ptr + ((size_t)seq * p.vt.heads * 64 + (col0 + u * 16 - p.vt.col0)) * p.vt.pitch + pos;
#pragma unroll
          for (int i = 0; i < 16; ++i) dst[(size_t)i * p.vt.pitch] = __float2bfloat16_rn(i & 1 ? f2_hi(y[i / 2]) : f2_lo(y[i / 2]));
        }
      };
      if (!RES && some) {                              // the box's last rows have been read out
        if (leader) bulk_wait_read<0>();
        __syncwarp();
      }
      if (some && col0 + 64 <= N) {                    // nearly all tiles
        uint32_t v[2][16];                             // one step ahead of the arithmetic
        tc_ld_32x16(taddr, v[0]);
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
          float s[16], b[16];
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            *reinterpret_cast<float4*>(s + i) = ldg4(ws + u * 16 + i);
            *reinterpret_cast<float4*>(b + i) = ldg4(bs + u * 16 + i);
          }
          tc_wait_ld_16(v[u & 1]);
          if (u < 3) tc_ld_32x16(taddr + (u + 1) * 16, v[(u + 1) & 1]); else release();
          sixteen(u, v[u & 1], s, b);
        }
      } else {
#pragma unroll 1
        for (uint32_t u = 0; some && u < 4 && col0 + u * 16 < N; ++u) {
          uint32_t v[16];
          tc_ld_32x16(taddr + u * 16, v);
          float s[16], b[16];
#pragma unroll
          for (uint32_t i = 0; i < 16; ++i) {          // (beyond the last column: its values again, whose results are dropped)
            const uint32_t c = min(u * 16 + i, N - 1 - col0);
            s[i] = __ldg(ws + c);
            b[i] = __ldg(bs + c);
          }
          tc_wait_ld_16(v);
          sixteen(u, v, s, b);
        }
        release();
      }
      if (some && !transposed) {
        const bool rest = N8 < N && N8 < col0 + 64;
        uint32_t w[4] = {0, 0, 0, 0};
        if (rest) put4(lds16(my_row ^ ((N8 - col0) / 8 << 4)), w);
        fence_async_smem();
        __syncwarp();
        if (whole_rows) {
          if (leader && col0 < N8) {
            tma_store_2d(&map_out, (int)col0, (int)row0, box);
            bulk_commit();
          }
          if (rest && row < M) {
            __nv_bfloat16* at = p.out + (long long)row * p.out_ld + N8;
#pragma unroll
            for (uint32_t i = 0; i < 7; ++i)
              if (N8 + i < N) at[i] = __ushort_as_bfloat16((unsigned short)(w[i / 2] >> (16 * (i & 1))));
          }
        } else {
          plain_box(p.out, p.out_ld, row0, col0, M, N, box, lane);
          fence_async_smem();
          __syncwarp();
        }
      }
      if (RES && leader) {
        bulk_wait_read<0>();
        fetch_residual(t + step);
      }
      __syncwarp();
    }
    if (leader) {
      bulk_wait_all();
      // a residual still on its way (only after a wait ran out) must land before the block ends
      volatile uint32_t never = 0;
      for (; r_used < r_issued; ++r_used) mbar_wait(res_bar(ew), r_used & 1u, &never, 200000000ull);
    }
  }

  __syncwarp();
  issued = __reduce_max_sync(0xFFFFFFFFu, issued);     // (the leader's)
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) {               // (pair: rank 0's barriers count both blocks' copies)
    const uint32_t back = issued < (uint32_t)S::STAGES ? issued : (uint32_t)S::STAGES;
    volatile uint32_t never = 0;
    for (uint32_t i = 0; i < back && rank == 0; ++i) {
      const uint32_t itx = issued - 1 - i;
      mbar_wait(full_bar(itx % S::STAGES), (itx / S::STAGES) & 1u, &never, 200000000ull);
    }
  }
  __syncthreads();
  __syncwarp();
  if constexpr (CTAS == 2) pair_meet();             // nobody reads or signals the other's memory any more
  if (warp == 1) {
    tc_fence_after();
    if constexpr (CTAS == 2)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(S::TMEM) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(S::TMEM) : "memory");
  }
}

namespace {
using DenseKernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const DenseArgs);

template <int CTAS, int BN, bool I8>
DenseKernel kernel_of(uint32_t act, bool res, bool vt) {
  if (vt) return !res && act == LAYER_ACT_NONE ? k_dense8_tc<CTAS, BN, I8, LAYER_ACT_NONE, false, true> : nullptr;
  switch (act) {
    case LAYER_ACT_NONE: return res ? k_dense8_tc<CTAS, BN, I8, LAYER_ACT_NONE, true, false> : k_dense8_tc<CTAS, BN, I8, LAYER_ACT_NONE, false, false>;
    case LAYER_ACT_GELU_ERF: return res ? k_dense8_tc<CTAS, BN, I8, LAYER_ACT_GELU_ERF, true, false> : k_dense8_tc<CTAS, BN, I8, LAYER_ACT_GELU_ERF, false, false>;
    case LAYER_ACT_GELU_TANH: return res ? k_dense8_tc<CTAS, BN, I8, LAYER_ACT_GELU_TANH, true, false> : k_dense8_tc<CTAS, BN, I8, LAYER_ACT_GELU_TANH, false, false>;
    default: return nullptr;
  }
}

// how many pairs of blocks the current device runs at a time (its SMs lie in groups, some with an odd number of them)
constexpr int MAX_DEVICES = 64;
int g_pairs[MAX_DEVICES];

template <int CTAS, int BN>
cudaLaunchConfig_t shape_config(cudaLaunchAttribute (&attr)[2], uint32_t grid, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(D8<CTAS, BN>::THREADS);
  cfg.dynamicSmemBytes = D8<CTAS, BN>::BYTES;
  cfg.stream = st;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = CTAS;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CTAS == 2 ? 2 : 1;
  return cfg;
}

template <int CTAS, int BN>
cudaError_t setup_shape() {
  for (uint32_t act = LAYER_ACT_NONE; act <= LAYER_ACT_GELU_TANH; ++act)
    for (int v = 0; v < 4; ++v) {
      const bool res = v & 1, vt = v & 2;
      for (const DenseKernel k : {kernel_of<CTAS, BN, true>(act, res, vt), kernel_of<CTAS, BN, false>(act, res, vt)}) {
        if (!k) continue;
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, D8<CTAS, BN>::BYTES);
        if (e != cudaSuccess) return e;
      }
    }
  return cudaSuccess;
}

// most: pairs or blocks that run at a time
template <int CTAS, int BN>
cudaError_t launch_shape(const DenseArgs& a, uint32_t most, cudaStream_t st) {
  const DenseKernel kern = a.format == LLMCACHE_I8 ? kernel_of<CTAS, BN, true>(a.act, a.residual != nullptr, a.vt.ptr != nullptr)
                                                   : kernel_of<CTAS, BN, false>(a.act, a.residual != nullptr, a.vt.ptr != nullptr);
  if (!kern) return cudaErrorInvalidValue;
  alignas(64) CUtensorMap map_a, map_w, map_out, map_res;
  if (!make_tensor_map_8bit(&map_a, a.a, a.m, a.k, a.a_ld, DM) || !make_tensor_map_8bit(&map_w, a.w, a.n, a.k, a.w_ld, BN / CTAS) ||
      !make_tensor_map_bf16_box64_pitch(&map_out, a.out, a.m, a.n >= 8 ? a.n & ~7u : 8u, a.out_ld))
    return cudaErrorInvalidValue;
  if (!a.residual) map_res = map_out;                  // (not used)
  else if (!make_tensor_map_bf16_box64_pitch(&map_res, a.residual, a.m, a.n, a.residual_ld)) return cudaErrorInvalidValue;
  const unsigned long long tiles = (unsigned long long)((a.m + CTAS * DM - 1) / (CTAS * DM)) * ((a.n + BN - 1) / BN);
  cudaLaunchAttribute attr[2];
  const cudaLaunchConfig_t cfg = shape_config<CTAS, BN>(attr, (tiles < most ? (uint32_t)tiles : most) * CTAS, st);
  return cudaLaunchKernelEx(&cfg, kern, map_a, map_w, map_out, map_res, a);
}
}  // namespace

cudaError_t setup_dense8_tc() {
  cudaError_t e = tensor_map_setup();
  if (e == cudaSuccess) e = setup_shape<2, 256>();
  if (e == cudaSuccess) e = setup_shape<1, 128>();
  if (e == cudaSuccess) e = setup_shape<1, 64>();
  if (e == cudaSuccess) e = setup_dense8_split();
  int dev = 0, pairs = 0;
  if (e == cudaSuccess) e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev < 0 || dev >= MAX_DEVICES)) e = cudaErrorInvalidDevice;
  if (e == cudaSuccess) {
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = shape_config<2, 256>(attr, 2, nullptr);
    cfg.attrs = attr + 1;                              // (the shape alone)
    cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&pairs, kernel_of<2, 256, true>(LAYER_ACT_NONE, false, false), &cfg);
  }
  if (e == cudaSuccess && pairs < 1) e = cudaErrorInvalidConfiguration;
  if (e == cudaSuccess) g_pairs[dev] = pairs;
  return e;
}

// What a form of the kernel takes, in us: `fixed` with the first tile's epilogue, a step for each 128 bytes of a tile's k, and for every further tile
// of a block as many steps again, or the epilogue where that is longer (`tile`, more with a residual).  A block's step is bound by its
// copies' rows of 128 bytes (0.8 ns each; 1.08 where rows do not start on 128 bytes, 1.5 where not on 32) or by its instructions.  Fitted, with all SMs at
// work, to products of 34 to 32,000 rows, 64 to 20,000 columns and k of 64 to 8,192, each timed in all forms; over 114 such products
// (profiles/eight_bit_forms.md) taking the least of these is 0.9 % above the best form of each, 34 % at worst (45 x 3,292 x 1,360: 52 clusters of 2 take
// 8.4 us, 128 x 64 6.2).  (The largest tile that gives every SM one, which was the rule before: 3,743 x 1,019 x 8,144 53 us where pairs take 34; 2,056 x 671 x
// 5,008 27 and 20.5 in 128 x 128; 2,500 x 2,304 x 768 13.5 and 11.2.)  The activation is left out (GELU adds 8 % to a
// pair's tile at k of 1,024).
struct FormTime { float fixed, instructions, tile, residual; };
constexpr FormTime T_PAIR{8.4f, 0.272f, 2.9f, 1.6f}, T_128{4.8f, 0.f, 2.2f, 0.8f}, T_64{3.9f, 0.19f, 1.7f, 0.45f};
constexpr FormTime T_SPLIT[3] = {{4.7f, 0.19f, 0.f, 0.f}, {4.75f, 0.19f, 0.f, 0.f}, {4.5f, 0.19f, 0.f, 0.f}};        // 2, 4, 8 blocks
float form_time(const DenseArgs& a, const FormTime& f, uint32_t rows_a, uint32_t rows_w, unsigned long long tiles, unsigned long long at_a_time, uint32_t steps) {
  auto row = [](long long ld) { return ld % 32 ? 1.5e-3f : ld % 128 ? 1.08e-3f : 0.8e-3f; };
  const float copies = rows_a * row(a.a_ld) + rows_w * row(a.w_ld), k = steps * (copies > f.instructions ? copies : f.instructions);
  // (a tile's steps and the epilogue of the one before run side by side, but not at full speed: 0.12 us for each step, fitted with the rest)
  const float further = f.tile + (a.residual ? f.residual : 0.f) + 0.12f * steps;
  return f.fixed + k + (float)((tiles + at_a_time - 1) / at_a_time - 1) * (k > further ? k : further);
}

DenseForm choose_dense8_tc(const DenseArgs& a, int dev, int sm_count) {
  const uint32_t steps = (a.k + DK - 1) / DK;
  const unsigned long long mb = (a.m + DM - 1) / DM, sms = (unsigned long long)sm_count, tiles64 = mb * ((a.n + 63) / 64);
  DenseForm best{0, form_time(a, T_PAIR, DM, 128, (mb + 1) / 2 * ((a.n + 255) / 256), (unsigned long long)g_pairs[dev], steps)};
  auto consider = [&](int form, float us) { if (us < best.us) best = DenseForm{form, us}; };
  consider(1, form_time(a, T_128, DM, 128, mb * ((a.n + 127) / 128), sms, steps));
  consider(2, form_time(a, T_64, DM, 64, tiles64, sms, steps));
  // clusters only where all tiles are at work at a time (a second wave costs more than it all), and every block has a step
  for (int i = 0; i < 3 && !a.vt.ptr; ++i) {
    const uint32_t parts = 2u << i;
    if (steps >= parts && tiles64 <= dense8_clusters(dev, parts)) consider(3 + i, form_time(a, T_SPLIT[i], DM, 64, 1, 1, (steps + parts - 1) / parts));
  }
  return best;
}

cudaError_t launch_dense8_tc(const DenseArgs& a, int form, int dev, int sm_count, cudaStream_t st) {
  switch (form) {
    case 0: return launch_shape<2, 256>(a, (uint32_t)g_pairs[dev], st);
    case 1: return launch_shape<1, 128>(a, (uint32_t)sm_count, st);
    case 2: return launch_shape<1, 64>(a, (uint32_t)sm_count, st);
    default: return launch_dense8_split(a, 2u << (form - 3), st);
  }
}

}  // namespace llmc
