// Arithmetic of the dense layers' epilogues, shared by the bf16 product (layer_gemm.cu) and the 8-bit ones (dense8_*.cu).
#pragma once
#include <cuda_bf16.h>
#include "ptx.cuh"

namespace llmc {

// GELU with the error function, x/2 + |x|/2 x erf(|x| / sqrt 2), for two values at once with packed fp32
// arithmetic and no special-function instruction: on u = min(|x|, 3.3 sqrt 2) an odd polynomial u Q(u^2) with nine
// coefficients stands for erf(u / sqrt 2) (beyond the clamp erf is within 3.1e-6 of its value there).  The
// coefficients minimise the largest error of GELU itself (gelu_erf_fit.py, beside this file): 8.2e-5 absolute
// with the float32 evaluation included, below the bf16 rounding of the result.  (The rational approximation with
// a reciprocal and an exponential used before cost two special-function instructions per element, and those
// bounded the epilogue of the first feed-forward product.)
__device__ __forceinline__ unsigned long long f2_dup(float x) { return f2_pack(x, x); }
// eight pairs at a time, stage by stage: the nine-term Horner chain of one pair is serial, eight of them side by
// side keep the pipeline fed with two epilogue warps per scheduler
__device__ __forceinline__ void gelu_erf2_x8(unsigned long long (&y)[8]) {
  unsigned long long u[8], s[8], q[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    u[j] = f2_pack(fminf(fabsf(f2_lo(y[j])), 4.666905f), fminf(fabsf(f2_hi(y[j])), 4.666905f));
    s[j] = f2_mul(u[j], u[j]);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) q[j] = f2_fma(f2_dup(4.615854921e-11f), s[j], f2_dup(-5.357377653e-09f));
  const float k[7] = {2.722534873e-07f, -8.016299034e-06f, 1.529819274e-04f, -2.011742676e-03f,
                      1.894705929e-02f, -1.315938234e-01f, 7.972128987e-01f};
#pragma unroll
  for (int t = 0; t < 7; ++t) {
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = f2_fma(q[j], s[j], f2_dup(k[t]));
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const unsigned long long erf_abs = f2_mul(u[j], q[j]);
    const unsigned long long h = f2_pack(0.5f * fabsf(f2_lo(y[j])), 0.5f * fabsf(f2_hi(y[j])));
    y[j] = f2_fma(h, erf_abs, f2_mul(y[j], f2_dup(0.5f)));
  }
}
__device__ __forceinline__ float gelu_tanh_f(float x) {
  return 0.5f * x * (1.0f + tanhf(0.7978845608028654f * (x + 0.044715f * x * x * x)));
}
// one value by the same operations in the same order: the same bits
__device__ __forceinline__ float gelu_erf_f(float x) {
  const float u = fminf(fabsf(x), 4.666905f), s = u * u;
  float q = fmaf(4.615854921e-11f, s, -5.357377653e-09f);
  const float k[7] = {2.722534873e-07f, -8.016299034e-06f, 1.529819274e-04f, -2.011742676e-03f,
                      1.894705929e-02f, -1.315938234e-01f, 7.972128987e-01f};
#pragma unroll
  for (int t = 0; t < 7; ++t) q = fmaf(q, s, k[t]);
  return fmaf(0.5f * fabsf(x), u * q, x * 0.5f);
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

}  // namespace llmc
