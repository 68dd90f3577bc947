// 8-bit operators (norm with an 8-bit output, product of two 8-bit matrices): shared declarations.
#pragma once
#include "layer.cuh"

namespace llmc {

enum { NORM_NONE = LLMCACHE_NORM_NONE, NORM_LAYER = LLMCACHE_NORM_LAYER, NORM_RMS = LLMCACHE_NORM_RMS };

// llmcache_norm_args, checked; leading dimensions in elements
struct NormArgs {
  const __nv_bfloat16 *x, *residual;
  __nv_bfloat16 *total, *out;
  const float *gain, *bias;
  uint8_t* q;
  float* scale;
  long long x_ld, residual_ld, total_ld, out_ld, q_ld;
  uint32_t n_rows, cols, kind, format;
  float eps;
  const uint32_t* count_dev;       // rows = min(n_rows, *count_dev * rows_per_count), or n_rows
  uint32_t rows_per_count;
};
cudaError_t setup_norm();
cudaError_t launch_norm(const NormArgs& a, int sm_count, cudaStream_t st);

// llmcache_dense_args, checked; leading dimensions in elements
struct DenseArgs {
  const uint8_t *a, *w;
  const float *a_scale, *w_scale, *bias;
  const __nv_bfloat16* residual;
  __nv_bfloat16* out;
  long long a_ld, w_ld, residual_ld, out_ld;
  uint32_t m, n, k, act, format;
  const uint32_t* count_dev;       // rows = min(m, *count_dev * rows_per_count), or m
  uint32_t rows_per_count;
  uint32_t* status;
  VtOut vt;                        // the layer's transposed V columns
};
// Sets the current device up for the operators with 8-bit values, on the first call: what launch_norm and launch_dense8 need.  Any thread may call it.
cudaError_t setup_eight();
cudaError_t setup_dense8_tc();
// the form of the tensor-core kernels that takes least, and what it takes; dev: the current device, which has been set up
struct DenseForm { int form; float us; };
DenseForm choose_dense8_tc(const DenseArgs& a, int dev, int sm_count);
cudaError_t launch_dense8_tc(const DenseArgs& a, int form, int dev, int sm_count, cudaStream_t st);
// k shared by clusters of 2, 4 or 8 blocks; how many of them run at a time on device dev, which has been set up
cudaError_t setup_dense8_split();
uint32_t dense8_clusters(int dev, uint32_t parts);
cudaError_t launch_dense8_split(const DenseArgs& a, uint32_t parts, cudaStream_t st);
// up to 32 rows
cudaError_t setup_dense8_few();
cudaError_t launch_dense8_few(const DenseArgs& a, int sm_count, cudaStream_t st);
cudaError_t launch_dense8(const DenseArgs& a, int sm_count, cudaStream_t st);

// rows of a call whose number may stand in device memory
__device__ __forceinline__ uint32_t rows_of(uint32_t most, const uint32_t* count_dev, uint32_t rows_per_count) {
  if (!count_dev) return most;
  const unsigned long long m = (unsigned long long)(*count_dev) * rows_per_count;
  return m < most ? (uint32_t)m : most;
}

}  // namespace llmc
