// Norm of a layer with the residual's addition in front and an output in 8 bits behind it:
//   h = x + residual;   y = h  |  (h - mean) rstd gain + bias  |  h / sqrt(mean(h^2) + eps) gain + bias
//   top = max |y| of the row;   scale = top / 127 (int8) or top / 448 (e4m3);   q = round(y / scale)
// h, y and the statistics are f32; h and y leave as bf16 where they are asked for.
//
// Bound by HBM: 2 bytes per element for each of x, residual, total and out that a call has, 1 for q, each moved once.  A
// row therefore stays in registers between its three reductions (mean, squares, largest magnitude).
#include <cuda_fp8.h>
#include "dense8.cuh"

namespace llmc {

namespace {

constexpr float NORM_TINY = 1e-30f;      // a row below this counts as zeros: its scale would lose its bits

// plain 16-byte load, kept in issue order.  (Not the read-only path: outputs may take the place of inputs row by row.)
__device__ __forceinline__ uint4 ld16(const void* p) {
  uint4 v;
  asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void add8(float (&h)[8], uint4 v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    h[2 * u] += __uint_as_float(w[u] << 16);
    h[2 * u + 1] += __uint_as_float(w[u] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint4 to_bf16(const float (&h)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(h[2 * u], h[2 * u + 1]);
    w[u] = *reinterpret_cast<const uint32_t*>(&v);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Quotients, not products with an inverse: values of few bits often lie halfway between two of the 8-bit ones, and only the
// correctly rounded quotient tells them apart from their neighbours.
__device__ __forceinline__ uint2 to_int8(const float (&y)[8], float scale) {
  uint32_t w[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = (uint32_t)__float2int_rn(y[4 * u + i] / scale) & 0xFFu;
    w[u] = b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
  }
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ uint2 to_e4m3(const float (&y)[8], float scale) {
  uint32_t w[2];
#pragma unroll
  for (int u = 0; u < 2; ++u)
    w[u] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(y[4 * u] / scale, y[4 * u + 1] / scale), __NV_SATFINITE, __NV_E4M3) |
           (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(y[4 * u + 2] / scale, y[4 * u + 3] / scale), __NV_SATFINITE, __NV_E4M3) << 16;
  return make_uint2(w[0], w[1]);
}

// Reductions over the TPR threads of a row: a warp, or a block whose warps meet in shared memory (slot: one of the three
// reductions of a row; every slot is read before the barrier of the next one, so a row's slots can be written again).
template <int TPR>
__device__ __forceinline__ float row_sum(float s, float* slot) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if constexpr (TPR > 32) {
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0.f;
#pragma unroll
    for (int i = 0; i < TPR / 32; ++i) s += slot[i];
  }
  return s;
}
template <int TPR>
__device__ __forceinline__ uint32_t row_max(uint32_t m, float* slot) {
  m = __reduce_max_sync(0xFFFFFFFFu, m);
  if constexpr (TPR > 32) {
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = __uint_as_float(m);
    __syncthreads();
    m = 0;
#pragma unroll
    for (int i = 0; i < TPR / 32; ++i) m = max(m, __float_as_uint(slot[i]));
  }
  return m;
}

// TPR threads per row, CH pieces of eight elements each
template <int TPR, int CH, int KIND>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR)
k_norm(const NormArgs a) {
  griddep_sync();
  constexpr uint32_t ROWS = TPR == 32 ? 8 : 1;             // rows of a block at a time
  __shared__ float slots[TPR > 32 ? 3 * (TPR / 32) : 1];
  float* const slot0 = slots;
  float* const slot1 = slots + (TPR > 32 ? TPR / 32 : 0);
  float* const slot2 = slots + (TPR > 32 ? 2 * (TPR / 32) : 0);
  const uint32_t rows = rows_of(a.n_rows, a.count_dev, a.rows_per_count);
  const uint32_t me = threadIdx.x % TPR, pieces = a.cols / 8;
  const float per = 1.0f / (float)a.cols;
  for (uint32_t row = blockIdx.x * ROWS + threadIdx.x / TPR; row < rows; row += gridDim.x * ROWS) {
    float h[CH][8];
    uint4 v[CH], r[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const uint32_t c = me + (uint32_t)i * TPR;
      v[i] = r[i] = make_uint4(0, 0, 0, 0);
      if (c < pieces) {
        v[i] = ld16(a.x + (long long)row * a.x_ld + c * 8);
        if (a.residual) r[i] = ld16(a.residual + (long long)row * a.residual_ld + c * 8);
      }
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
#pragma unroll
      for (int u = 0; u < 8; ++u) h[i][u] = 0.f;
      add8(h[i], v[i]);
      if (a.residual) add8(h[i], r[i]);
    }
    if (a.total) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const uint32_t c = me + (uint32_t)i * TPR;
        if (c < pieces) st_stream16(a.total + (long long)row * a.total_ld + c * 8, to_bf16(h[i]));
      }
    }
    if constexpr (KIND != NORM_NONE) {
      float mu = 0.f;
      if constexpr (KIND == NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
          for (int u = 0; u < 8; ++u) s += h[i][u];
        mu = row_sum<TPR>(s, slot0) * per;
      }
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        if (KIND == NORM_RMS || me + (uint32_t)i * TPR < pieces) {
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            h[i][u] -= mu;
            s = fmaf(h[i][u], h[i][u], s);
          }
        }
      }
      const float rstd = 1.0f / sqrtf(row_sum<TPR>(s, slot1) * per + a.eps);
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const uint32_t c = me + (uint32_t)i * TPR;
        if (c < pieces) {
          float g[8], b[8];
          const float4 one = make_float4(1.f, 1.f, 1.f, 1.f), zero = make_float4(0.f, 0.f, 0.f, 0.f);
          *reinterpret_cast<float4*>(g) = a.gain ? __ldg(reinterpret_cast<const float4*>(a.gain + c * 8)) : one;
          *reinterpret_cast<float4*>(g + 4) = a.gain ? __ldg(reinterpret_cast<const float4*>(a.gain + c * 8 + 4)) : one;
          *reinterpret_cast<float4*>(b) = a.bias ? __ldg(reinterpret_cast<const float4*>(a.bias + c * 8)) : zero;
          *reinterpret_cast<float4*>(b + 4) = a.bias ? __ldg(reinterpret_cast<const float4*>(a.bias + c * 8 + 4)) : zero;
#pragma unroll
          for (int u = 0; u < 8; ++u) h[i][u] = fmaf(h[i][u] * rstd, g[u], b[u]);
        }
      }
    }
    if (a.out) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const uint32_t c = me + (uint32_t)i * TPR;
        if (c < pieces) st_stream16(a.out + (long long)row * a.out_ld + c * 8, to_bf16(h[i]));
      }
    }
    if (a.q) {
      // magnitudes compared as integers: infinities are above all numbers, and NaN above them
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int u = 0; u < 8; ++u) m = max(m, __float_as_uint(h[i][u]) & 0x7FFFFFFFu);
      m = row_max<TPR>(m, slot2);
      const bool bad = m >= 0x7F800000u;
      const float top = __uint_as_float(m);
      const float scale = bad ? __uint_as_float(0x7FC00000u) : top < NORM_TINY ? 0.f : top / (a.format == LLMCACHE_I8 ? 127.f : 448.f);
      if (me == 0) a.scale[row] = scale;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const uint32_t c = me + (uint32_t)i * TPR;
        if (c < pieces) {
          const uint2 e = !(scale > 0.f) ? make_uint2(0, 0) : a.format == LLMCACHE_I8 ? to_int8(h[i], scale) : to_e4m3(h[i], scale);
          *reinterpret_cast<uint2*>(a.q + (long long)row * a.q_ld + c * 8) = e;
        }
      }
    }
    // rows with a single reduction: its slot may be written again only when all have read it
    if (TPR > 32 && (KIND == NORM_NONE || (KIND == NORM_RMS && !a.q))) __syncthreads();
  }
}

template <int TPR, int KIND>
cudaError_t launch_width(const NormArgs& a, uint32_t ch, int sm_count, cudaStream_t st) {
  constexpr uint32_t ROWS = TPR == 32 ? 8 : 1, THREADS = TPR == 32 ? 256 : TPR;
  const unsigned long long cap = (unsigned long long)sm_count * (2048 / THREADS);
  unsigned long long blocks = ((unsigned long long)a.n_rows + ROWS - 1) / ROWS;
  if (blocks > cap) blocks = cap;
  auto kern = ch <= 1 ? k_norm<TPR, 1, KIND> : ch == 2 ? k_norm<TPR, 2, KIND> : ch == 3 ? k_norm<TPR, 3, KIND> : k_norm<TPR, 4, KIND>;
  return launch_k(kern, dim3((uint32_t)blocks), dim3(THREADS), 0, st, a);
}

template <int KIND>
cudaError_t launch_kind(const NormArgs& a, int sm_count, cudaStream_t st) {
  // up to four pieces of eight elements per thread
  const uint32_t pieces = a.cols / 8;
  auto per = [&](uint32_t threads) { return (pieces + threads - 1) / threads; };
  if (pieces <= 32 * 4) return launch_width<32, KIND>(a, per(32), sm_count, st);
  if (pieces <= 128 * 4) return launch_width<128, KIND>(a, per(128), sm_count, st);
  return launch_width<512, KIND>(a, per(512), sm_count, st);
}

}  // namespace

cudaError_t launch_norm(const NormArgs& a, int sm_count, cudaStream_t st) {
  if (a.n_rows == 0) return cudaSuccess;
  switch (a.kind) {
    case NORM_NONE: return launch_kind<NORM_NONE>(a, sm_count, st);
    case NORM_LAYER: return launch_kind<NORM_LAYER>(a, sm_count, st);
    case NORM_RMS: return launch_kind<NORM_RMS>(a, sm_count, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace llmc
