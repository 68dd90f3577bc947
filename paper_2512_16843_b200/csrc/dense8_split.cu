// Product of two 8-bit matrices (dense8_tc.cu) with a long k and too few tiles for all SMs: a cluster of 2, 4 or 8 blocks shares the k of a
// tile of 128 x 64.  A block alone takes 0.19 us for each 128 bytes of k, however many others there are.  Every block sums its part of k into tensor
// memory; then each takes a share of the columns, to which the others send their sums through the cluster's shared memory.  They are added in the order of
// k: integers exactly, fp32 in a fixed order.  512 rows, 512 columns, k of 4,096: 10.0 us without, 8.0 with clusters of 2, 6.8 with 4; 448
// columns of 128 rows 5.4 with 8; 512 rows, 1,024 columns 10.1 and 8.3.  All that the results need besides their sums is asked for while these are
// formed, and eight warps share them (four, asking behind the sums: 9.6, 7.6, 6.0 and 9.9 us).
// All mbarrier waits are bounded (status word); the blocks meet twice, at points that every one reaches whatever its waits gave.
#include <cuda.h>
#include "dense8.cuh"
#include "layer_epi.cuh"

namespace llmc {

namespace {
constexpr int SM_ROWS = 128, SN = 64, SK = 128, S_STAGES = 6, S_THREADS = 320;      // warp 0: TMA, warp 1: MMA, eight warps for the sums
constexpr uint32_t SA_BYTES = SM_ROWS * SK, SB_BYTES = SN * SK;
struct SplitSmem {
  static constexpr uint32_t A = 0;
  static constexpr uint32_t B = A + S_STAGES * SA_BYTES;
  static constexpr uint32_t EX = B + S_STAGES * SB_BYTES;           // sums sent here: [block][four columns of this block][row]: a warp's stores are 512 bytes in a row
  static constexpr uint32_t SCALE = EX + SM_ROWS * SN * 4;            // of this block's columns, then their biases
  static constexpr uint32_t BAR = SCALE + 2 * SN / 2 * 4;
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
// bf16 at p, or 0 where it is not there
__device__ __forceinline__ uint32_t one_bf16(const __nv_bfloat16* p, bool there) { return there ? __bfloat16_as_ushort(*p) : 0u; }
__device__ __forceinline__ void st_cluster16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
}  // namespace

// PARTS blocks per tile
template <bool I8, uint32_t PARTS>
__global__ void __launch_bounds__(S_THREADS, 1)
k_dense8_split(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_w, const DenseArgs p) {
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
  const uint32_t NB = (N + SN - 1) / SN, tile = blockIdx.x / PARTS, mb = tile / NB, nb = tile % NB;
  const uint32_t KB = (p.k + SK - 1) / SK, kb0 = KB * rank / PARTS, kb1 = KB * (rank + 1) / PARTS;
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
  cluster_arrive();                                     // (this block runs: its shared memory may be written from now on)
  const uint32_t tmem = *tmem_slot;

  uint32_t issued = 0;
  const bool leader = elect_one();
  if (work && warp == 0) {
    if (leader && !producer_idle(p.status)) {
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
    if (leader) {
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
  // What the results need besides their sums comes while these are formed: scales and biases of this block's columns into shared
  // memory, a row's scale and residual into registers.  Two threads share a row.
  constexpr uint32_t EACH = SN / PARTS, MINE = EACH / 2;           // columns of a block, of a thread
  const uint32_t quarter = warp & 3u, half = (warp - 2) >> 2, row_in_tile = quarter * 32 + lane, row = mb * SM_ROWS + row_in_tile;
  const uint32_t first = rank * EACH, c0 = half * MINE, col0 = nb * SN + first + c0;
  float* const w_scale = reinterpret_cast<float*>(gbase + S::SCALE);
  float* const bias = w_scale + SN / 2;
  float sa = 0.f;
  uint2 residual[MINE / 4];
  if (work && warp >= 2) {
    if (half == 0 && row_in_tile < EACH) {              // (beyond the last column: its values again, whose results are dropped)
      const uint32_t c = min(nb * SN + first + row_in_tile, N - 1);
      w_scale[row_in_tile] = p.w_scale[c];
      bias[row_in_tile] = p.bias ? p.bias[c] : 0.f;
    }
    sa = row < M ? p.a_scale[row] : 0.f;
#pragma unroll
    for (uint32_t i = 0; i < MINE / 4; ++i) {
      residual[i] = make_uint2(0, 0);
      const uint32_t col = col0 + i * 4;
      if (!p.residual || row >= M || col >= N) continue;
      const __nv_bfloat16* from = p.residual + (long long)row * p.residual_ld + col;
      if (col + 4 <= N) residual[i] = *reinterpret_cast<const uint2*>(from);
      else residual[i] = make_uint2(one_bf16(from, true) | one_bf16(from + 1, col + 1 < N) << 16, one_bf16(from + 2, col + 2 < N));
    }
  }
  __syncwarp();
  cluster_wait();                                       // all blocks of the cluster run
  if (work && warp >= 2) {
    const bool live = __all_sync(0xFFFFFFFFu, mbar_wait(sums_bar, 0u, abort_flag, lim));
    if (!live) { *abort_flag = 1; atomicExch(p.status, 1u); }
    tc_fence_after();
#pragma unroll
    for (uint32_t u = 0; live && u < SN / 32; ++u) {
      const uint32_t c16 = half * (SN / 2) + u * 16;
      uint32_t v[16];
      tc_ld_32x16(tmem + c16 + ((quarter * 32u) << 16), v);
      tc_wait_ld_16(v);
#pragma unroll
      for (uint32_t q = 0; q < 16; q += 4) {
        const uint32_t c = c16 + q;
        st_cluster16(of_rank(base + S::EX + ((rank * EACH + c % EACH) / 4 * SM_ROWS + row_in_tile) * 16, c / EACH), v[q], v[q + 1], v[q + 2], v[q + 3]);
      }
    }
    tc_fence_before();
  }
  __syncwarp();
  pair_meet();                                          // all sums have arrived
  if (work && warp >= 2 && row < M) {
#pragma unroll
    for (uint32_t g = 0; g < MINE / 4; ++g) {
      const uint32_t c = c0 + g * 4, col = col0 + g * 4;
      if (col >= N) break;
      float f[4] = {0.f, 0.f, 0.f, 0.f};
      uint32_t s[4] = {0, 0, 0, 0};
#pragma unroll
      for (uint32_t b = 0; b < PARTS; ++b) {
        const uint4 x = lds16(base + S::EX + ((b * EACH + c) / 4 * SM_ROWS + row_in_tile) * 16);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (I8) s[i] += w[i];                         // (two's complement)
          else f[i] += __uint_as_float(w[i]);
        }
      }
      const uint32_t res[2] = {residual[g].x, residual[g].y};
      uint32_t o[4];
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) {
        const float r = __uint_as_float(i & 1 ? res[i / 2] & 0xFFFF0000u : res[i / 2] << 16);
        // the same operations as in dense8_tc.cu
        float v = I8 ? (float)(int32_t)s[i] : f[i];
        v = fmaf(__fmul_rn(v, sa), w_scale[c + i], bias[c + i]);
        if (p.act == LAYER_ACT_NONE) v = p.residual ? __fadd_rn(v, r) : v;
        else {
          const float phi = p.act == LAYER_ACT_GELU_ERF ? gelu_phi_f<false>(v) : gelu_phi_f<true>(v);
          v = p.residual ? fmaf(v, phi, r) : __fmul_rn(v, phi);
        }
        o[i] = __bfloat16_as_ushort(__float2bfloat16_rn(v));
      }
      __nv_bfloat16* to = p.out + (long long)row * p.out_ld + col;
      if (col + 4 <= N) {
        *reinterpret_cast<uint2*>(to) = make_uint2(o[0] | o[1] << 16, o[2] | o[3] << 16);
      } else {
#pragma unroll
        for (uint32_t i = 0; i < 3; ++i)
          if (col + i < N) to[i] = __ushort_as_bfloat16((unsigned short)o[i]);
      }
    }
  }

  __syncwarp();
  issued = __reduce_max_sync(0xFFFFFFFFu, issued);      // (the leader's)
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

using SplitKernel = void (*)(const CUtensorMap, const CUtensorMap, const DenseArgs);
SplitKernel split_kernel(bool i8, uint32_t parts) {
  switch (parts) {
    case 2: return i8 ? k_dense8_split<true, 2> : k_dense8_split<false, 2>;
    case 4: return i8 ? k_dense8_split<true, 4> : k_dense8_split<false, 4>;
    default: return i8 ? k_dense8_split<true, 8> : k_dense8_split<false, 8>;
  }
}

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
  cudaError_t e = cudaSuccess;
  for (uint32_t parts = 2; parts <= 8; parts *= 2)
    for (const bool i8 : {true, false})
      if (e == cudaSuccess) e = cudaFuncSetAttribute(split_kernel(i8, parts), cudaFuncAttributeMaxDynamicSharedMemorySize, SplitSmem::BYTES);
  int dev = 0;
  if (e == cudaSuccess) e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev < 0 || dev >= MAX_DEVICES)) e = cudaErrorInvalidDevice;
  for (int i = 0; i < 3 && e == cudaSuccess; ++i) {
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = split_config(attr, 2u << i, 2u << i, nullptr);
    cfg.numAttrs = 1;                                   // (the shape alone)
    e = cudaOccupancyMaxActiveClusters(&g_clusters[dev][i], split_kernel(true, 2u << i), &cfg);
  }
  return e;
}

uint32_t dense8_clusters(int dev, uint32_t parts) { return (uint32_t)g_clusters[dev][parts == 2 ? 0 : parts == 4 ? 1 : 2]; }

cudaError_t launch_dense8_split(const DenseArgs& a, uint32_t parts, cudaStream_t st) {
  alignas(64) CUtensorMap map_a, map_w;
  if (!make_tensor_map_8bit(&map_a, a.a, a.m, a.k, a.a_ld, SM_ROWS) || !make_tensor_map_8bit(&map_w, a.w, a.n, a.k, a.w_ld, SN))
    return cudaErrorInvalidValue;
  cudaLaunchAttribute attr[2];
  const cudaLaunchConfig_t cfg = split_config(attr, (a.m + SM_ROWS - 1) / SM_ROWS * ((a.n + SN - 1) / SN) * parts, parts, st);
  return cudaLaunchKernelEx(&cfg, split_kernel(a.format == LLMCACHE_I8, parts), map_a, map_w, a);
}

}  // namespace llmc
