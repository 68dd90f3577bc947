// Product of two 8-bit matrices for few rows of activations (next tokens): out[m, n] as in dense8_tc.cu, m <= 32.
//
// The weights are read once and nothing else is large, so the kernel is a stream of weights through registers: a warp takes 16 output
// channels and a share of k, in pieces of 64 bytes, with several pieces' loads in flight.  mma.sync m16n8k32 sums with the channels as the rows of the product and
// tokens as its columns, eight at a time: a tensor-memory tile would be 128 tokens high and wait for a ring of copies to fill.  A
// lane loads 16 neighbouring bytes of a channel and of a token where the instruction's layout names four words that are 16 bytes
// apart: the sum over k does not depend on its order as long as both operands have the same one.  The warps' sums meet in shared memory;
// integers have one sum in any order, fp32 sums are added in the order of the warps.
#include "dense8.cuh"
#include "layer_epi.cuh"

namespace llmc {

namespace {

constexpr uint32_t FEW_CH = 16;                     // output channels of a block

template <bool I8>
__device__ __forceinline__ void mma8(uint32_t (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (I8)
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 ldw(const uint8_t* p, bool there) {
  return there ? ld_nc16(p) : make_uint4(0, 0, 0, 0);
}

// NT groups of eight tokens; a block's warps share the k of its channels
template <int NT, bool I8>
__global__ void __launch_bounds__(512) k_dense8_few(const DenseArgs p) {
  griddep_sync();
  extern __shared__ uint32_t sums[];                // [warps][NT * 8 tokens][FEW_CH]
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const uint32_t g = lane >> 2, t = lane & 3u;
  const uint32_t M = rows_of(p.m, p.count_dev, p.rows_per_count);
  if (M == 0) return;
  const uint32_t n0 = blockIdx.x * FEW_CH;
  // channels and tokens beyond the ends read the last one's bytes; what comes of them is dropped
  const uint8_t* w0 = p.w + (long long)min(n0 + g, p.n - 1) * p.w_ld + t * 16;
  const uint8_t* w1 = p.w + (long long)min(n0 + g + 8, p.n - 1) * p.w_ld + t * 16;
  const uint8_t* x[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) x[i] = p.a + (long long)min((uint32_t)i * 8 + g, M - 1) * p.a_ld + t * 16;
  uint32_t c[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) c[i][j] = 0;         // (zero bits are 0.0 too)
  constexpr uint32_t EACH = NT * 8 * FEW_CH;          // sums of a warp
  // what the first result of this thread needs besides its sum, on its way behind the first weights (for eight tokens: 2,304 x 768 2.3 ->
  // 2.0 us, 1,024 x 4,096 4.2 -> 2.9; with more of them it costs registers that the loads need)
  constexpr bool AHEAD = NT == 1;
  float sa_first = 0.f, sw_first = 0.f, b_first = 0.f, r_first = 0.f;
  constexpr int U = NT <= 2 ? 4 : 2;                 // pieces of k in flight
  const uint32_t pieces = (p.k + 63) / 64;
  for (uint32_t kb = warp; kb < pieces; kb += warps * U) {
    uint4 a[U], b[U], y[U][NT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t k = (kb + u * warps) * 64;
      const bool there = k + t * 16 < p.k;            // k is a multiple of 16
      a[u] = ldw(w0 + k, there);
      b[u] = ldw(w1 + k, there);
#pragma unroll
      for (int i = 0; i < NT; ++i) y[u][i] = ldw(x[i] + k, there);
    }
    if (AHEAD && kb == warp) {
      const uint32_t m = threadIdx.x / FEW_CH, n = n0 + threadIdx.x % FEW_CH;
      if (threadIdx.x < EACH && m < M && n < p.n) {
        sa_first = p.a_scale[m];
        sw_first = p.w_scale[n];
        if (p.bias) b_first = p.bias[n];
        if (p.residual) r_first = __bfloat162float(p.residual[(long long)m * p.residual_ld + n]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        mma8<I8>(c[i], a[u].x, b[u].x, a[u].y, b[u].y, y[u][i].x, y[u][i].y);
        mma8<I8>(c[i], a[u].z, b[u].z, a[u].w, b[u].w, y[u][i].z, y[u][i].w);
      }
  }
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)                       // row of the product: g or g + 8; column: 2 t or 2 t + 1
      sums[(warp * NT * 8 + i * 8 + 2 * t + (j & 1)) * FEW_CH + g + (j >> 1) * 8] = c[i][j];
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < EACH; e += blockDim.x) {
    const uint32_t m = e / FEW_CH, n = n0 + e % FEW_CH;
    if (m >= M || n >= p.n) continue;
    const uint32_t* from = sums + e;
    float v;
    if constexpr (I8) {
      int32_t s = 0;
      for (uint32_t w = 0; w < warps; ++w) s += (int32_t)from[w * EACH];
      v = (float)s;
    } else {
      v = 0.f;
      for (uint32_t w = 0; w < warps; ++w) v += __uint_as_float(from[w * EACH]);
    }
    // the same operations as in dense8_tc.cu
    const bool is_first = AHEAD && e == threadIdx.x && warp < pieces;      // (a warp without a piece has not looked)
    const float sa = is_first ? sa_first : p.a_scale[m], sw = is_first ? sw_first : p.w_scale[n];
    const float b = is_first ? b_first : p.bias ? p.bias[n] : 0.f;
    const float r = is_first ? r_first : p.residual ? __bfloat162float(p.residual[(long long)m * p.residual_ld + n]) : 0.f;
    v = fmaf(__fmul_rn(v, sa), sw, b);
    if (p.act == LAYER_ACT_NONE) v = p.residual ? __fadd_rn(v, r) : v;
    else {
      const float phi = p.act == LAYER_ACT_GELU_ERF ? gelu_phi_f<false>(v) : gelu_phi_f<true>(v);
      v = p.residual ? fmaf(v, phi, r) : __fmul_rn(v, phi);
    }
    p.out[(long long)m * p.out_ld + n] = __float2bfloat16_rn(v);
  }
}

template <int NT>
void (*kernel_for(bool i8))(const DenseArgs) { return i8 ? k_dense8_few<NT, true> : k_dense8_few<NT, false>; }

template <int NT>
cudaError_t launch_tokens(const DenseArgs& a, int sm_count, cudaStream_t st) {
  const uint32_t pieces = (a.k + 63) / 64, channels = (a.n + FEW_CH - 1) / FEW_CH;
  // three pieces of k or more for a warp, up to 8 warps; 16 only where the channels do not fill the SMs (8,192 x 8,192: 17 us
  // with 16, 15 with 8)
  const uint32_t most = channels * 8ull >= 24ull * (uint32_t)sm_count ? 8 : 16;
  const uint32_t want = pieces < 4 ? pieces : pieces < 16 ? 4 : pieces < 64 ? 8 : 16, warps = want < most ? want : most;
  const size_t smem = (size_t)warps * NT * 8 * FEW_CH * 4;
  return launch_k(kernel_for<NT>(a.format == LLMCACHE_I8), dim3(channels), dim3(warps * 32), smem, st, a);
}

}  // namespace

// The kernels are loaded with the others' set-up, not with the first call that takes them, which may stand in a capture.
cudaError_t setup_dense8_few() {
  cudaFuncAttributes f;
  for (const bool i8 : {true, false})
    for (auto k : {kernel_for<1>(i8), kernel_for<2>(i8), kernel_for<4>(i8)}) {
      const cudaError_t e = cudaFuncGetAttributes(&f, k);
      if (e != cudaSuccess) return e;
    }
  return cudaSuccess;
}

cudaError_t launch_dense8_few(const DenseArgs& a, int sm_count, cudaStream_t st) {
  if (a.m <= 8) return launch_tokens<1>(a, sm_count, st);
  if (a.m <= 16) return launch_tokens<2>(a, sm_count, st);
  return a.m <= 32 ? launch_tokens<4>(a, sm_count, st) : cudaErrorInvalidValue;
}

}  // namespace llmc
