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
// GELU for the 8-bit products, whose epilogues have half the time of the bf16 ones: x phi(x), phi(x) = x Q(x^2) + 1/2 clamped to
// [0, 1] by the multiply-add itself, Q with nine coefficients (gelu_fit.py, beside this file).  The largest error is 3.8e-5 (erf) and
// 2.9e-5 (tanh) for all arguments: Q's last coefficient is positive, so beyond the fitted range the polynomial leaves [0, 1] on the
// right side.  What is added behind it (a residual) joins the last multiplication.  12 instructions per pair where the form above takes 16 (tanhf: two special-function instructions per element and
// more arithmetic than all else in an epilogue).
template <bool TANH>
__device__ __forceinline__ constexpr float gelu_coef(int i) {
  constexpr float erf_form[9] = {4.197455578e-11f, -4.249007368e-09f, 1.902243838e-07f, -5.006177162e-06f, 8.711776172e-05f,
                                 -1.071386971e-03f, 9.695150889e-03f, -6.615559757e-02f, 3.988020718e-01f};
  constexpr float tanh_form[9] = {5.853447588e-11f, -5.609957388e-09f, 2.374260362e-07f, -5.902364137e-06f, 9.717926878e-05f,
                                  -1.137998188e-03f, 9.932884946e-03f, -6.649324298e-02f, 3.988072276e-01f};
  return TANH ? tanh_form[i] : erf_form[i];
}
// two neighbouring bf16
__device__ __forceinline__ unsigned long long bf16_pair(uint32_t w) {
  return f2_pack(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <bool TANH, bool ADD>
__device__ __forceinline__ void gelu_phi2_x8(unsigned long long (&y)[8], const uint32_t (&add)[8]) {
  unsigned long long s[8], q[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) s[j] = f2_mul(y[j], y[j]);
#pragma unroll
  for (int j = 0; j < 8; ++j) q[j] = f2_fma(f2_dup(gelu_coef<TANH>(0)), s[j], f2_dup(gelu_coef<TANH>(1)));
#pragma unroll
  for (int t = 2; t < 9; ++t) {
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = f2_fma(q[j], s[j], f2_dup(gelu_coef<TANH>(t)));
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const unsigned long long phi = f2_pack(__saturatef(fmaf(f2_lo(q[j]), f2_lo(y[j]), 0.5f)), __saturatef(fmaf(f2_hi(q[j]), f2_hi(y[j]), 0.5f)));
    y[j] = ADD ? f2_fma(y[j], phi, bf16_pair(add[j])) : f2_mul(y[j], phi);
  }
}
// phi of one value by the same operations in the same order: the same bits
template <bool TANH>
__device__ __forceinline__ float gelu_phi_f(float x) {
  const float s = __fmul_rn(x, x);
  float q = fmaf(gelu_coef<TANH>(0), s, gelu_coef<TANH>(1));
#pragma unroll
  for (int t = 2; t < 9; ++t) q = fmaf(q, s, gelu_coef<TANH>(t));
  return __saturatef(fmaf(q, x, 0.5f));
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

}  // namespace llmc
