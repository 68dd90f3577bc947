// Product of two 8-bit matrices on the tensor cores:
//   out[m, n] = act(a_scale[m] w_scale[n] sum_k a[m, k] w[n, k] + bias[n]) (+ residual[m, n]),   bf16 out
// int8 is summed in 32-bit integers (exact: k <= 131,056), e4m3 in fp32.  Tiles of 128 rows x BN columns x 128 bytes of k come by
// TMA (128-byte swizzle, zeros beyond the matrices' ends) into a ring, tcgen05.mma 128 x BN x 32 sums them in one of two
// accumulators in tensor memory, and eight epilogue warps drain the other meanwhile: scales, bias, activation, residual; rows
// leave and residuals arrive through boxes of 32 rows x 32 columns per warp that the bulk-copy engine moves.
// The number of valid rows may come from device memory.  All mbarrier waits are bounded (status word).
#include <cuda.h>
#include "dense8.cuh"
#include "layer_epi.cuh"

namespace llmc {

namespace {
constexpr int DM = 128, DK = 128;
constexpr int D_THREADS = 320;                      // warp 0: TMA, warp 1: MMA, warps 2..9: epilogue (two sets of four)
constexpr int D_EPI = 256;
constexpr uint32_t DA_BYTES = DM * DK;
constexpr uint32_t D_BOX = 32 * 64;                 // a warp's 32 rows of a 32-column group

template <int BN>
struct D8 {
  static constexpr int STAGES = BN == 256 ? 4 : BN == 128 ? 5 : 7;
  static constexpr uint32_t B_BYTES = BN * DK;
  static constexpr uint32_t A = 0;
  static constexpr uint32_t B = A + STAGES * DA_BYTES;
  static constexpr uint32_t STG = B + STAGES * B_BYTES;          // one box per epilogue warp on its way out
  static constexpr uint32_t RES = STG + 8 * D_BOX;               // the same for the residual on its way in
  static constexpr uint32_t COL = RES + 8 * D_BOX;               // float w_scale [BN], float bias [BN]
  static constexpr uint32_t BAR = COL + BN * 8;
  static constexpr uint32_t MISC = BAR + (2 * STAGES + 12) * 8;
  static constexpr uint32_t BYTES = MISC + 64;
  static constexpr uint32_t TMEM = 2 * BN;
  static_assert(BYTES <= 232448, "shared memory of one block");
};
}  // namespace

// I8: int8 or e4m3; ACT, RES, VT as in the bf16 product: each epilogue carries only its own code
template <int BN, bool I8, uint32_t ACT, bool RES, bool VT>
__global__ void __launch_bounds__(D_THREADS, 1)
k_dense8_tc(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_w,
            const __grid_constant__ CUtensorMap map_out, const __grid_constant__ CUtensorMap map_res, const DenseArgs p) {
  griddep_sync();
  using S = D8<BN>;
  extern __shared__ __align__(1024) uint8_t gbase[];   // (the swizzle counts from multiples of 1,024 bytes; there is no room to round up)
  const uint32_t base = smem_u32(gbase);
  if (base & 1023u) {
    if (threadIdx.x == 0) atomicExch(p.status, 1u);
    return;
  }
  const uint32_t sA = base + S::A, sB = base + S::B;
  float* scol = reinterpret_cast<float*>(gbase + S::COL);
  const uint32_t bar0 = base + S::BAR;
  auto full_bar = [&](uint32_t s) { return bar0 + 8 * s; };
  auto empty_bar = [&](uint32_t s) { return bar0 + 8 * (S::STAGES + s); };
  auto tfull_bar = [&](uint32_t b) { return bar0 + 8 * (2 * S::STAGES + b); };
  auto tempty_bar = [&](uint32_t b) { return bar0 + 8 * (2 * S::STAGES + 2 + b); };
  auto res_bar = [&](uint32_t w) { return bar0 + 8 * (2 * S::STAGES + 4 + w); };      // one per epilogue warp
  volatile uint32_t* misc = reinterpret_cast<volatile uint32_t*>(gbase + S::MISC);
  volatile uint32_t* tmem_slot = misc + 0;
  volatile uint32_t* abort_flag = misc + 1;
  volatile uint32_t* epi_go = misc + 2;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned long long lim = wait_limit(p.status);

  const uint32_t M = rows_of(p.m, p.count_dev, p.rows_per_count), N = p.n;
  const uint32_t KB = (p.k + DK - 1) / DK;
  const uint32_t MB = (M + DM - 1) / DM, NB = (N + BN - 1) / BN;
  const uint32_t n_tiles = MB * NB;

  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < (uint32_t)S::STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (uint32_t b = 0; b < 2; ++b) {
      mbar_init(tfull_bar(b), 1);
      mbar_init(tempty_bar(b), D_EPI);
    }
    for (uint32_t w = 0; w < D_EPI / 32; ++w) mbar_init(res_bar(w), 1);
    misc[1] = 0; misc[2] = 0; misc[3] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32((const void*)tmem_slot)), "r"(S::TMEM) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  uint32_t issued = 0;
  if (warp == 0) {
    if (lane == 0 && !producer_idle(p.status)) {       // ---- TMA producer
      bool ok = true;
      for (uint32_t t = blockIdx.x; t < n_tiles && ok; t += gridDim.x) {
        const uint32_t mb = t / NB, nb = t % NB;       // consecutive blocks share the A tile in L2
        for (uint32_t kb = 0; kb < KB; ++kb) {
          const uint32_t s = issued % S::STAGES, ph = (issued / S::STAGES) & 1u;
          if (!mbar_wait(empty_bar(s), ph ^ 1u, abort_flag, lim)) { ok = false; break; }
          mbar_expect_tx(full_bar(s), DA_BYTES + S::B_BYTES);
          tma_load_2d(sA + s * DA_BYTES, &map_a, (int)(kb * DK), (int)(mb * DM), full_bar(s));
          tma_load_2d(sB + s * S::B_BYTES, &map_w, (int)(kb * DK), (int)(nb * BN), full_bar(s));
          ++issued;
        }
      }
      if (!ok) { *abort_flag = 1; atomicExch(p.status, 1u); }
    }
  } else if (warp == 1) {
    if (lane == 0) {                                   // ---- MMA issuer
      // operand types: signed 8-bit integers into 32-bit ones, or e4m3 into fp32
      constexpr uint32_t idesc = (I8 ? (2u << 4) | (1u << 7) | (1u << 10) : (1u << 4)) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(DM >> 4) << 24);
      bool ok = true;
      uint32_t it = 0, tile = 0;
      for (uint32_t t = blockIdx.x; t < n_tiles && ok; t += gridDim.x, ++tile) {
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
            if (I8) tc_mma_i8(d_tmem, da + kk * 2, db + kk * 2, idesc, (kb | kk) != 0u);
            else    tc_mma_f8(d_tmem, da + kk * 2, db + kk * 2, idesc, (kb | kk) != 0u);
          }
          tc_commit(empty_bar(s));
        }
        if (ok) tc_commit(tfull_bar(buf));
      }
      if (!ok) { *abort_flag = 1; atomicExch(p.status, 1u); }
    }
  } else {
    // ---- epilogue: thread = one row of the tile, 32 columns at a time; set 0 takes the even groups, set 1 the odd ones.
    // Rows of a partial block of a device-counted M, ragged last columns and transposed V columns use plain stores.
    const uint32_t et = threadIdx.x - 64, set = et >> 7, quarter = warp & 3u, ew = et >> 5;
    const uint32_t box = ew * D_BOX;
    const uint32_t row_in_tile = quarter * 32 + lane;
    const uint32_t my_off = box + lane * 64u, sw = (lane >> 1) & 3u;
    // Tiles that leave through the boxes: what they have beyond the last row is cut off by the copy.  Columns are cut off in
    // pieces of 16 bytes only: a last group that ends inside one uses plain stores.
    auto boxed = [&](uint32_t t) { return M == p.m || (t / NB + 1) * DM <= M; };
    const uint32_t n_boxed = N % 8 ? N / 32 * 32 : N;
    uint32_t r_issued = 0, r_used = 0;
    uint32_t ct = blockIdx.x, cg = set;                // next residual rows to request (lane 0 of every warp)
    auto res_issue = [&]() {
      while (ct < n_tiles && (!boxed(ct) || (ct % NB) * BN + cg * 32 >= n_boxed)) { ct += gridDim.x; cg = set; }
      if (ct >= n_tiles) return;
      const uint32_t cmb = ct / NB, cnb = ct % NB;
      mbar_expect_tx(res_bar(ew), D_BOX);
      tma_load_2d(base + S::RES + box, &map_res, (int)(cnb * BN + cg * 32), (int)(cmb * DM + quarter * 32), res_bar(ew));
      ++r_issued;
      cg += 2;
      if (cg >= BN / 32 || cnb * BN + cg * 32 >= n_boxed) { cg = set; ct += gridDim.x; }
    };
    if (RES && lane == 0) res_issue();
    uint32_t tile = 0;
    for (uint32_t t = blockIdx.x; t < n_tiles; t += gridDim.x, ++tile) {
      const uint32_t mb = t / NB, nb = t % NB;
      const uint32_t buf = tile & 1u, bph = (tile >> 1) & 1u;
      for (uint32_t x = et; x < (uint32_t)BN; x += D_EPI) {
        const uint32_t c = nb * BN + x;
        scol[x] = c < N ? p.w_scale[c] : 0.f;
        scol[BN + x] = (p.bias && c < N) ? p.bias[c] : 0.f;
      }
      const uint32_t row = mb * DM + row_in_tile;
      const bool row_ok = row < M, tile_boxed = boxed(t);
      const float sa = row_ok ? p.a_scale[row] : 0.f;
      if (et == 0) *epi_go = *abort_flag;
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (*epi_go) break;
      // a wait that ran out ends the warp's work on the tile: nothing is read, and nothing asked for that is not waited for
      bool live = __all_sync(0xFFFFFFFFu, mbar_wait(tfull_bar(buf), bph, abort_flag, lim));
      if (!live) { *abort_flag = 1; atomicExch(p.status, 1u); }
      tc_fence_after();
      const uint32_t taddr = tmem_base + buf * BN + ((quarter * 32u) << 16);
      const unsigned long long sa2 = f2_pack(sa, sa);
#pragma unroll 1
      for (uint32_t c = set * 32; live && c < (uint32_t)BN; c += 64) {
        const uint32_t col0 = nb * BN + c;
        if (col0 >= N) break;
        const bool staged = tile_boxed && col0 < n_boxed;
        if (RES && staged) {
          live = __all_sync(0xFFFFFFFFu, mbar_wait(res_bar(ew), r_used & 1u, abort_flag, lim));
          if (!live) { *abort_flag = 1; atomicExch(p.status, 1u); break; }
          ++r_used;
        }
        uint32_t v[32];
        tc_ld_32x32(taddr + c, v);
        // the residual of this group goes to registers first and its box is refilled at once, so that the next
        // group's residual has this whole group's time to arrive
        uint4 rr[4];
        if (RES && staged) {
          const uint8_t* rb = gbase + S::RES + my_off;
#pragma unroll
          for (uint32_t q = 0; q < 4; ++q) rr[q] = *reinterpret_cast<const uint4*>(rb + ((q ^ sw) << 4));
          __syncwarp();
          if (lane == 0) res_issue();
        }
        tc_wait_ld();
        float f[32];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const float2* s2 = reinterpret_cast<const float2*>(scol + c) + half * 8;
          const float2* b2 = reinterpret_cast<const float2*>(scol + BN + c) + half * 8;
          unsigned long long y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float2 s = s2[j], b = b2[j];
            const uint32_t v0 = v[half * 16 + 2 * j], v1 = v[half * 16 + 2 * j + 1];
            const unsigned long long x = I8 ? f2_pack((float)(int32_t)v0, (float)(int32_t)v1)
                                            : f2_pack(__uint_as_float(v0), __uint_as_float(v1));
            y[j] = f2_fma(f2_mul(x, sa2), f2_pack(s.x, s.y), f2_pack(b.x, b.y));
          }
          if (ACT == LAYER_ACT_GELU_ERF) gelu_erf2_x8(y);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            f[half * 16 + 2 * j] = f2_lo(y[j]);
            f[half * 16 + 2 * j + 1] = f2_hi(y[j]);
          }
        }
        if (ACT == LAYER_ACT_GELU_TANH) {
#pragma unroll
          for (int i = 0; i < 32; ++i) f[i] = gelu_tanh_f(f[i]);
        }
        if (VT && col0 >= p.vt.col0) {
          // the V third of a q|k|v product, transposed per head (see the bf16 product)
          if (row_ok) {
            const uint32_t seq = row / p.rows_per_count, pos = row - seq * p.rows_per_count;
            __nv_bfloat16* dst = p.vt.ptr + ((size_t)seq * p.vt.heads * 64 + (col0 - p.vt.col0)) * p.vt.pitch + pos;
#pragma unroll
            for (int i = 0; i < 32; ++i) dst[(size_t)i * p.vt.pitch] = __float2bfloat16_rn(f[i]);
          }
          continue;
        }
        if (staged) {
          if (RES) {
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q) {
              const uint32_t w[4] = {rr[q].x, rr[q].y, rr[q].z, rr[q].w};
#pragma unroll
              for (int u = 0; u < 4; ++u) {
                f[q * 8 + 2 * u]     += __uint_as_float(w[u] << 16);
                f[q * 8 + 2 * u + 1] += __uint_as_float(w[u] & 0xFFFF0000u);
              }
            }
          }
          if (lane == 0) bulk_wait_read<0>();           // the warp's previous rows have been read out
          __syncwarp();
          uint8_t* ob = gbase + S::STG + my_off;
#pragma unroll
          for (uint32_t q = 0; q < 4; ++q)
            *reinterpret_cast<uint4*>(ob + ((q ^ sw) << 4)) =
                make_uint4(pack_bf16(f[q * 8], f[q * 8 + 1]), pack_bf16(f[q * 8 + 2], f[q * 8 + 3]),
                           pack_bf16(f[q * 8 + 4], f[q * 8 + 5]), pack_bf16(f[q * 8 + 6], f[q * 8 + 7]));
          fence_async_smem();
          __syncwarp();
          if (lane == 0) {
            tma_store_2d(&map_out, (int)col0, (int)(mb * DM + quarter * 32), base + S::STG + box);
            bulk_commit();
          }
        } else if (row_ok) {
          const __nv_bfloat16* r = RES ? p.residual + (size_t)row * p.residual_ld + col0 : nullptr;
          __nv_bfloat16* o = p.out + (size_t)row * p.out_ld + col0;
#pragma unroll
          for (uint32_t i = 0; i < 32; ++i)
            if (col0 + i < N) o[i] = __float2bfloat16_rn(RES ? f[i] + __bfloat162float(r[i]) : f[i]);
        }
      }
      tc_fence_before();
      mbar_arrive(tempty_bar(buf));
      asm volatile("bar.sync 1, 256;" ::: "memory");   // the scales and biases of the next tile overwrite this one's
    }
    if (lane == 0) {
      bulk_wait_all();
      // residual boxes still on their way (only after a wait ran out): they must land before the block ends
      volatile uint32_t never = 0;
      for (; r_used < r_issued; ++r_used) mbar_wait(res_bar(ew), r_used & 1u, &never, 200000000ull);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) {
    const uint32_t back = issued < (uint32_t)S::STAGES ? issued : (uint32_t)S::STAGES;
    volatile uint32_t never = 0;
    for (uint32_t i = 0; i < back; ++i) {
      const uint32_t itx = issued - 1 - i;
      mbar_wait(full_bar(itx % S::STAGES), (itx / S::STAGES) & 1u, &never, 200000000ull);
    }
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(S::TMEM) : "memory");
  }
}

namespace {
using DenseKernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const DenseArgs);

template <int BN, bool I8>
DenseKernel kernel_of(uint32_t act, bool res, bool vt) {
  if (vt) return !res && act == LAYER_ACT_NONE ? k_dense8_tc<BN, I8, LAYER_ACT_NONE, false, true> : nullptr;
  switch (act) {
    case LAYER_ACT_NONE: return res ? k_dense8_tc<BN, I8, LAYER_ACT_NONE, true, false> : k_dense8_tc<BN, I8, LAYER_ACT_NONE, false, false>;
    case LAYER_ACT_GELU_ERF: return res ? k_dense8_tc<BN, I8, LAYER_ACT_GELU_ERF, true, false> : k_dense8_tc<BN, I8, LAYER_ACT_GELU_ERF, false, false>;
    case LAYER_ACT_GELU_TANH: return res ? k_dense8_tc<BN, I8, LAYER_ACT_GELU_TANH, true, false> : k_dense8_tc<BN, I8, LAYER_ACT_GELU_TANH, false, false>;
    default: return nullptr;
  }
}

template <int BN>
cudaError_t setup_width() {
  for (uint32_t act = LAYER_ACT_NONE; act <= LAYER_ACT_GELU_TANH; ++act)
    for (int v = 0; v < 4; ++v) {
      const bool res = v & 1, vt = v & 2;
      for (const DenseKernel k : {kernel_of<BN, true>(act, res, vt), kernel_of<BN, false>(act, res, vt)}) {
        if (!k) continue;
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, D8<BN>::BYTES);
        if (e != cudaSuccess) return e;
      }
    }
  return cudaSuccess;
}

template <int BN>
cudaError_t launch_width(const DenseArgs& a, int sm_count, cudaStream_t st) {
  const DenseKernel kern = a.format == LLMCACHE_I8 ? kernel_of<BN, true>(a.act, a.residual != nullptr, a.vt.ptr != nullptr)
                                                   : kernel_of<BN, false>(a.act, a.residual != nullptr, a.vt.ptr != nullptr);
  if (!kern) return cudaErrorInvalidValue;
  alignas(64) CUtensorMap map_a, map_w, map_out, map_res;
  if (!make_tensor_map_8bit(&map_a, a.a, a.m, a.k, a.a_ld, DM) || !make_tensor_map_8bit(&map_w, a.w, a.n, a.k, a.w_ld, BN) ||
      !make_tensor_map_bf16_box32_pitch(&map_out, a.out, a.m, a.n, a.out_ld) ||
      !make_tensor_map_bf16_box32_pitch(&map_res, a.residual ? a.residual : a.out, a.m, a.n, a.residual ? a.residual_ld : a.out_ld))
    return cudaErrorInvalidValue;
  const unsigned long long tiles = (unsigned long long)((a.m + DM - 1) / DM) * ((a.n + BN - 1) / BN);
  const uint32_t grid = tiles < (unsigned long long)sm_count ? (uint32_t)tiles : (uint32_t)sm_count;
  return launch_k(kern, dim3(grid), dim3(D_THREADS), D8<BN>::BYTES, st, map_a, map_w, map_out, map_res, a);
}
}  // namespace

cudaError_t setup_dense8_tc() {
  cudaError_t e = tensor_map_setup();
  if (e == cudaSuccess) e = setup_width<256>();
  if (e == cudaSuccess) e = setup_width<128>();
  if (e == cudaSuccess) e = setup_width<64>();
  return e;
}

cudaError_t launch_dense8_tc(const DenseArgs& a, int sm_count, cudaStream_t st) {
  // the widest tile that gives every SM one
  const unsigned long long mb = (a.m + DM - 1) / DM;
  if (mb * ((a.n + 255) / 256) >= (unsigned long long)sm_count) return launch_width<256>(a, sm_count, st);
  if (mb * ((a.n + 127) / 128) >= (unsigned long long)sm_count) return launch_width<128>(a, sm_count, st);
  return launch_width<64>(a, sm_count, st);
}

}  // namespace llmc
