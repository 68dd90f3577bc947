// Product of two 8-bit matrices (dense8_tc.cu) with a long k and too few tiles for all SMs: a cluster of 2, 4 or 8 blocks shares the k of a
// tile of 128 x 64.  A block alone is bound by its own copies, about 58 bytes per cycle, 24 KB for each 128 bytes of k (1,024
// columns, k of 4,096: 12.4 us whatever the number of rows up to 1,000; asking for all of it ahead in the second-level cache made it
// 17).  With a cluster of 4 8.4 us; 2,048 columns, k of 8,192 21.2 -> 11.3.  Every block sums its part of k into tensor memory; then each takes a share of the columns, to which the others send their sums
// through the cluster's shared memory.  They are added in the order of k: integers exactly, fp32 in a fixed order.
// All mbarrier waits are bounded (status word); the blocks meet twice, at points that every one reaches whatever its waits gave.
#include <cuda.h>
#include "dense8.cuh"
#include "layer_epi.cuh"

namespace llmc {

namespace {
constexpr int SM_ROWS = 128, SN = 64, SK = 128, S_STAGES = 6, S_THREADS = 192;      // warp 0: TMA, warp 1: MMA, four warps for the sums
constexpr uint32_t SA_BYTES = SM_ROWS * SK, SB_BYTES = SN * SK;
struct SplitSmem {
  static constexpr uint32_t A = 0;
  static constexpr uint32_t B = A + S_STAGES * SA_BYTES;
  static constexpr uint32_t EX = B + S_STAGES * SB_BYTES;           // sums sent here: [block][four columns of this block][row]: a warp's stores are 512 bytes in a row
  static constexpr uint32_t BAR = EX + SM_ROWS * SN * 4;
  static constexpr uint32_t MISC = BAR + (2 * S_STAGES + 1) * 8;
  static constexpr uint32_t BYTES = MISC + 16 + 1024;
};
static_assert(SplitSmem::BYTES <= 232448, "shared memory of one block");

// a shared-memory address of another block of the cluster
__device__ __forceinline__ uint32_t of_rank(uint32_t saddr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr), "r"(rank));
  return r;
}
__device__ __forceinline__ void st_cluster16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
}  // namespace

template <bool I8>
__global__ void __launch_bounds__(S_THREADS, 1)
k_dense8_split(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_w, const DenseArgs p, uint32_t parts) {
  griddep_sync();
  using S = SplitSmem;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;           // (the same in all blocks of a cluster)
  uint8_t* gbase = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bar0 = base + S::BAR;
  auto full_bar = [&](uint32_t s) { return bar0 + 8 * s; };
  auto empty_bar = [&](uint32_t s) { return bar0 + 8 * (S_STAGES + s); };
  const uint32_t sums_bar = bar0 + 8 * (2 * S_STAGES);
  volatile uint32_t* misc = reinterpret_cast<volatile uint32_t*>(gbase + S::MISC);
  volatile uint32_t* tmem_slot = misc + 0;
  volatile uint32_t* abort_flag = misc + 1;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = pair_rank();
  const unsigned long long lim = wait_limit(p.status);

  const uint32_t M = rows_of(p.m, p.count_dev, p.rows_per_count), N = p.n;
  const uint32_t NB = (N + SN - 1) / SN, tile = blockIdx.x / parts, mb = tile / NB, nb = tile % NB;
  const uint32_t KB = (p.k + SK - 1) / SK, kb0 = KB * rank / parts, kb1 = KB * (rank + 1) / parts;
  const bool work = mb * SM_ROWS < M;                  // the same for the whole cluster

  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < (uint32_t)S_STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    mbar_init(sums_bar, 1);
    misc[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32((const void*)tmem_slot)), "r"((uint32_t)SN) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  uint32_t issued = 0;
  if (work && warp == 0) {
    if (lane == 0 && !producer_idle(p.status)) {
      bool ok = true;
      for (uint32_t kb = kb0; kb < kb1; ++kb) {
        const uint32_t s = issued % S_STAGES, ph = (issued / S_STAGES) & 1u;
        if (!mbar_wait(empty_bar(s), ph ^ 1u, abort_flag, lim)) { ok = false; break; }
        mbar_expect_tx(full_bar(s), SA_BYTES + SB_BYTES);
        tma_load_2d(base + S::A + s * SA_BYTES, &map_a, (int)(kb * SK), (int)(mb * SM_ROWS), full_bar(s));
        tma_load_2d(base + S::B + s * SB_BYTES, &map_w, (int)(kb * SK), (int)(nb * SN), full_bar(s));
        ++issued;
      }
      if (!ok) { *abort_flag = 1; atomicExch(p.status, 1u); }
    }
  } else if (work && warp == 1) {
    if (lane == 0) {
      constexpr uint32_t idesc = (I8 ? (2u << 4) | (1u << 7) | (1u << 10) : (1u << 4)) | ((uint32_t)(SN >> 3) << 17) | ((uint32_t)(SM_ROWS >> 4) << 24);
      bool ok = true;
      for (uint32_t it = 0; it < kb1 - kb0; ++it) {
        const uint32_t s = it % S_STAGES, ph = (it / S_STAGES) & 1u;
        if (!mbar_wait(full_bar(s), ph, abort_flag, lim)) { ok = false; break; }
        tc_fence_after();
        const uint64_t da = smem_desc_sw128(base + S::A + s * SA_BYTES), db = smem_desc_sw128(base + S::B + s * SB_BYTES);
#pragma unroll
        for (uint32_t kk = 0; kk < SK / 32; ++kk) {
          if (I8) tc_mma_i8(tmem, da + kk * 2, db + kk * 2, idesc, (it | kk) != 0u);
          else    tc_mma_f8(tmem, da + kk * 2, db + kk * 2, idesc, (it | kk) != 0u);
        }
        tc_commit(empty_bar(s));
      }
      if (ok) tc_commit(sums_bar);
      else { *abort_flag = 1; atomicExch(p.status, 1u); }
    }
  }
  __syncwarp();
  pair_meet();                                          // (all blocks of the cluster run: their shared memory may be written)
  const uint32_t quarter = warp & 3u, row_in_tile = quarter * 32 + lane, each = SN / parts;     // columns of a block
  if (work && warp >= 2) {
    const bool live = __all_sync(0xFFFFFFFFu, mbar_wait(sums_bar, 0u, abort_flag, lim));
    if (!live) { *abort_flag = 1; atomicExch(p.status, 1u); }
    tc_fence_after();
#pragma unroll
    for (uint32_t u = 0; live && u < SN / 16; ++u) {
      uint32_t v[16];
      tc_ld_32x16(tmem + u * 16 + ((quarter * 32u) << 16), v);
      tc_wait_ld_16(v);
#pragma unroll
      for (uint32_t q = 0; q < 16; q += 4) {
        const uint32_t c = u * 16 + q;                  // (a block has 8 columns or more)
        st_cluster16(of_rank(base + S::EX + ((rank * each + c % each) / 4 * SM_ROWS + row_in_tile) * 16, c / each), v[q], v[q + 1], v[q + 2], v[q + 3]);
      }
    }
    tc_fence_before();
  }
  __syncwarp();
  pair_meet();                                          // all sums have arrived
  const uint32_t row = mb * SM_ROWS + row_in_tile;
  if (work && warp >= 2 && row < M) {
    const float sa = p.a_scale[row];
    for (uint32_t c = 0; c < each; c += 8) {
      const uint32_t col = nb * SN + rank * each + c;
      if (col >= N) break;
      const bool whole = col + 8 <= N;
      float f[8];
      uint32_t s[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) { s[i] = 0; f[i] = 0.f; }
      for (uint32_t b = 0; b < parts; ++b) {
        const uint32_t at = base + S::EX + ((b * each + c) / 4 * SM_ROWS + row_in_tile) * 16;
        const uint4 x = lds16(at), y = lds16(at + SM_ROWS * 16);
        const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (I8) s[i] += w[i];                         // (two's complement)
          else f[i] += __uint_as_float(w[i]);
        }
      }
      uint32_t res[4] = {0, 0, 0, 0}, o[8];
      if (p.residual) {
        const __nv_bfloat16* from = p.residual + (long long)row * p.residual_ld + col;
        if (whole) {
          const uint4 r = *reinterpret_cast<const uint4*>(from);
          res[0] = r.x; res[1] = r.y; res[2] = r.z; res[3] = r.w;
        } else {
#pragma unroll
          for (uint32_t i = 0; i < 8; ++i)
            if (col + i < N) res[i / 2] |= (uint32_t)__bfloat16_as_ushort(from[i]) << (16 * (i & 1));
        }
      }
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) {
        const bool there = whole || col + i < N;
        const float r = __uint_as_float(i & 1 ? res[i / 2] & 0xFFFF0000u : res[i / 2] << 16);
        // the same operations as in dense8_tc.cu
        float v = I8 ? (float)(int32_t)s[i] : f[i];
        v = fmaf(__fmul_rn(v, sa), there ? p.w_scale[col + i] : 0.f, there && p.bias ? p.bias[col + i] : 0.f);
        if (p.act == LAYER_ACT_NONE) v = p.residual ? __fadd_rn(v, r) : v;
        else {
          const float phi = p.act == LAYER_ACT_GELU_ERF ? gelu_phi_f<false>(v) : gelu_phi_f<true>(v);
          v = p.residual ? fmaf(v, phi, r) : __fmul_rn(v, phi);
        }
        o[i] = __bfloat16_as_ushort(__float2bfloat16_rn(v));
      }
      __nv_bfloat16* to = p.out + (long long)row * p.out_ld + col;
      if (whole) {
        *reinterpret_cast<uint4*>(to) = make_uint4(o[0] | o[1] << 16, o[2] | o[3] << 16, o[4] | o[5] << 16, o[6] | o[7] << 16);
      } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
          if (col + i < N) to[i] = __ushort_as_bfloat16((unsigned short)o[i]);
      }
    }
  }

  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) {               // copies in flight must land before shared memory is released
    const uint32_t back = issued < (uint32_t)S_STAGES ? issued : (uint32_t)S_STAGES;
    volatile uint32_t never = 0;
    for (uint32_t i = 0; i < back; ++i) {
      const uint32_t x = issued - 1 - i;
      mbar_wait(full_bar(x % S_STAGES), (x / S_STAGES) & 1u, &never, 200000000ull);
    }
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)SN) : "memory");
  }
}

namespace {
// how many clusters of 2, 4 and 8 blocks each device runs at a time (its SMs lie in groups that clusters do not leave)
constexpr int MAX_DEVICES = 64;
int g_clusters[MAX_DEVICES][3];

cudaLaunchConfig_t split_config(cudaLaunchAttribute (&attr)[2], uint32_t grid, uint32_t parts, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(S_THREADS);
  cfg.dynamicSmemBytes = SplitSmem::BYTES;
  cfg.stream = st;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = parts;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cfg;
}
}  // namespace

cudaError_t setup_dense8_split() {
  cudaError_t e = cudaFuncSetAttribute(k_dense8_split<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, SplitSmem::BYTES);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(k_dense8_split<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, SplitSmem::BYTES);
  int dev = 0;
  if (e == cudaSuccess) e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev < 0 || dev >= MAX_DEVICES)) e = cudaErrorInvalidDevice;
  for (int i = 0; i < 3 && e == cudaSuccess; ++i) {
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = split_config(attr, 2u << i, 2u << i, nullptr);
    cfg.numAttrs = 1;                                   // (the shape alone)
    e = cudaOccupancyMaxActiveClusters(&g_clusters[dev][i], k_dense8_split<true>, &cfg);
  }
  return e;
}

uint32_t dense8_split_parts(const DenseArgs& a) {
  int dev = 0;
  if (a.vt.ptr || cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return 1;
  const unsigned long long tiles = (unsigned long long)((a.m + SM_ROWS - 1) / SM_ROWS) * ((a.n + SN - 1) / SN);
  const uint32_t KB = (a.k + SK - 1) / SK;
  // The largest cluster with which all tiles are at work at a time (a second wave costs more than it all), where k is long: meeting and
  // sending costs about 3.5 us, a step of k 0.23 us (1,024 columns: k of 4,096 12.4 us alone, 8.4 with 4 blocks; k of 1,024 5.6 and 6.6).
  for (int i = 2; i >= 0 && KB >= SPLIT_LEAST; --i)
    if (tiles <= (unsigned long long)g_clusters[dev][i]) return 2u << i;
  return 1;
}

cudaError_t launch_dense8_split(const DenseArgs& a, uint32_t parts, cudaStream_t st) {
  alignas(64) CUtensorMap map_a, map_w;
  if (!make_tensor_map_8bit(&map_a, a.a, a.m, a.k, a.a_ld, SM_ROWS) || !make_tensor_map_8bit(&map_w, a.w, a.n, a.k, a.w_ld, SN))
    return cudaErrorInvalidValue;
  cudaLaunchAttribute attr[2];
  const cudaLaunchConfig_t cfg = split_config(attr, (a.m + SM_ROWS - 1) / SM_ROWS * ((a.n + SN - 1) / SN) * parts, parts, st);
  return cudaLaunchKernelEx(&cfg, a.format == LLMCACHE_I8 ? k_dense8_split<true> : k_dense8_split<false>, map_a, map_w, a, parts);
}

}  // namespace llmc
