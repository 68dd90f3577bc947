// Norm of a layer with the residual's addition in front and an output in 8 bits behind it:
//   h = x + residual;   y = h  |  (h - mean) rstd gain + bias  |  h / sqrt(mean(h^2) + eps) gain + bias
//   top = max |y| of the row;   scale = top / 127 (int8) or top / 448 (e4m3);   q = round(y / scale)
// h, y and the statistics are f32; h and y leave as bf16 where they are asked for.
//
// Bound by HBM: 2 bytes per element for each of x, residual, total and out that a call has, 1 for q, each moved once.  A
// row therefore stays in registers between its three reductions (mean, squares, largest magnitude).  131,072 x 1,024 with residual and total to e4m3 takes
// 144 us (6.5 TB/s), 98,304 x 768 layer norm to bf16 and int8 69 (5.5), 131,072 x 1,024 rms to bf16 alone 91 (5.9), 4,001 x 4,096 to e4m3 10.0 (4.9),
// 12,288 x 768 layer norm to bf16 and int8 11.7 (4.0; 9.9 where part of it lies in L2).
//
// Where little is moved per element the work per row counts: its reductions are a chain, and the rows that an SM has registers for do not
// cover it.  105 M elements of 1,024 columns from bf16 to int8 take 52 us without a norm and 76 with rms (48 are the bytes' time), of 2,048
// 75, of 5,000 90; 2,988 x 9,272 18, 27 with rms and 42 with a residual and layer norm (12.7 and, with the residual, 21.1; see STAGED).
#include <cuda_fp8.h>
#include "dense8.cuh"
#include "ptx.cuh"

namespace llmc {

namespace {

constexpr int MAX_DEVICES = 64;
constexpr float NORM_TINY = 1e-30f;      // a row below this counts as zeros: its scale would lose its bits

// plain 16-byte load, kept in issue order.  (Not the read-only path: outputs may take the place of inputs row by row.)
__device__ __forceinline__ uint4 ld16(const void* p) {
  uint4 v;
  asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}
// the same into shared memory while the thread goes on; not `there`: zeros
__device__ __forceinline__ void ld16_async(uint32_t to, const void* p, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(p), "r"(there ? 16u : 0u) : "memory");
}
__device__ __forceinline__ void ld16_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
typedef unsigned long long f2;           // two neighbouring columns in f32
__device__ __forceinline__ f2 bf16_2(uint32_t w) { return f2_pack(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
__device__ __forceinline__ uint32_t to_bf16(f2 v) {
  const __nv_bfloat162 o = __floats2bfloat162_rn(f2_lo(v), f2_hi(v));
  return *reinterpret_cast<const uint32_t*>(&o);
}
__device__ __forceinline__ uint4 to_bf16x8(const f2 (&h)[4]) { return make_uint4(to_bf16(h[0]), to_bf16(h[1]), to_bf16(h[2]), to_bf16(h[3])); }
// the larger magnitude; NaN if there is one
__device__ __forceinline__ float max_nan(float m, f2 v) {
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(m), "f"(fabsf(f2_lo(v))), "f"(fabsf(f2_hi(v))));
  return m;
}
// y / scale, correctly rounded.  Quotients, not products with an inverse: values of few bits often lie halfway between two of
// the 8-bit ones, and only the rounded quotient tells them apart from their neighbours.  Markstein's correction (IBM Journal of Research
// and Development 34, 1990): with inv the rounded inverse of the scale and q = y inv, q + (y - q scale) inv is the rounded quotient,
// the difference being exact in a fused multiply-add.  (Where it underflows, y is far below half a step.)  Three instructions for two
// values; a division takes about ten for each, which took more time than the memory.
__device__ __forceinline__ f2 quotient(f2 y, f2 inv, f2 minus_scale) {
  const f2 q = f2_mul(y, inv);
  return f2_fma(f2_fma(q, minus_scale, y), inv, q);
}
// Integers of up to 2^22 in magnitude added to 1.5 2^23 stand in the low bits of the sum, rounded to the nearest even one.
__device__ __forceinline__ uint2 to_int8(const f2 (&y)[4], f2 inv, f2 minus_scale) {
  uint32_t w[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const f2 magic = f2_pack(12582912.f, 12582912.f);
    const f2 a = f2_add(quotient(y[2 * u], inv, minus_scale), magic), b = f2_add(quotient(y[2 * u + 1], inv, minus_scale), magic);
    w[u] = __byte_perm(__byte_perm((uint32_t)a, (uint32_t)(a >> 32), 0x0040), __byte_perm((uint32_t)b, (uint32_t)(b >> 32), 0x0040), 0x5410);
  }
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ uint32_t e4m3_2(f2 v) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(f2_lo(v), f2_hi(v)), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint2 to_e4m3(const f2 (&y)[4], f2 inv, f2 minus_scale) {
  uint32_t w[2];
#pragma unroll
  for (int u = 0; u < 2; ++u)
    w[u] = e4m3_2(quotient(y[2 * u], inv, minus_scale)) | e4m3_2(quotient(y[2 * u + 1], inv, minus_scale)) << 16;
  return make_uint2(w[0], w[1]);
}

// Reductions over the TPR threads of a row: a part of a warp, a warp, or a block whose warps meet in shared memory (slot: one of
// the three reductions of a row; every slot is read before the barrier of the next one, so a row's slots can be written again).
template <int TPR>
__device__ __forceinline__ float row_sum(float s, float* slot) {
#pragma unroll
  for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
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
  if constexpr (TPR >= 32) {
    m = __reduce_max_sync(0xFFFFFFFFu, m);
  } else {
#pragma unroll
    for (int o = TPR / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  }
  if constexpr (TPR > 32) {
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = __uint_as_float(m);
    __syncthreads();
    m = 0;
#pragma unroll
    for (int i = 0; i < TPR / 32; ++i) m = max(m, __float_as_uint(slot[i]));
  }
  return m;
}

// threads and rows of a block
template <int TPR>
struct Shape {
  static constexpr uint32_t THREADS = TPR <= 32 ? 128 : TPR, ROWS = THREADS / TPR;
};

// Pieces of eight elements that a thread of a row's TPR may have.  At least: fewer would leave as many threads idle as half of them with twice
// the pieces, and the choice takes those (launch_kind).
template <int TPR>
constexpr uint32_t LEAST_CH = TPR == 8 ? 1 : TPR <= 64 ? 2 : 3;
template <int TPR>
constexpr uint32_t MOST_CH = TPR <= 32 ? 3 : TPR == 256 ? 8 : 4;

// Rows of 256 threads with four pieces each and more: their next row waits in shared memory, each thread's pieces in its own place, so that
// registers are left for more blocks, that is more rows on their way through the reductions at a time.
template <int TPR, uint32_t CH>
constexpr bool STAGED = TPR == 256 && CH >= 4;
// blocks per SM that the registers are to be enough for (0: as many as come of it)
template <int TPR, uint32_t CH>
constexpr int BLOCKS = !STAGED<TPR, CH> ? (TPR == 256 ? 2 : 0) : CH <= 6 ? 3 : 2;

// TPR threads per row, CH pieces of eight elements each.  A thread's columns are the same in every row, so gains and biases stay in
// registers where there is room for them (KEEP): read again for every row they keep the first-level cache busy for longer than the row takes
// (1,536 columns, rms without residual: 94 us per 105 M elements, 73 with KEEP).
template <int TPR, uint32_t CH, int KIND>
__global__ void __launch_bounds__(Shape<TPR>::THREADS, (BLOCKS<TPR, CH>))
k_norm(const NormArgs a) {
  griddep_sync();
  constexpr uint32_t ROWS = Shape<TPR>::ROWS;
  constexpr bool KEEP = KIND != NORM_NONE && TPR <= 256 && !STAGED<TPR, CH>;
  __shared__ float slots[TPR > 32 ? 3 * (TPR / 32) : 1];
  float* const slot0 = slots;
  float* const slot1 = slots + (TPR > 32 ? TPR / 32 : 0);
  float* const slot2 = slots + (TPR > 32 ? 2 * (TPR / 32) : 0);
  const uint32_t rows = rows_of(a.n_rows, a.count_dev, a.rows_per_count);
  const uint32_t me = threadIdx.x % TPR, pieces = a.cols / 8;
  const float per = 1.0f / (float)a.cols;
  extern __shared__ __align__(16) uint8_t stage[];      // a thread's pieces of its next row; the residual's behind all threads'
  const uint32_t mine = STAGED<TPR, CH> ? smem_u32(stage) + threadIdx.x * 16 : 0u;
  uint4 v[STAGED<TPR, CH> ? 1 : CH], r[STAGED<TPR, CH> ? 1 : CH];
  auto fetch = [&](uint32_t row) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const uint32_t c = me + (uint32_t)i * TPR;
      const bool there = c < pieces && row < rows;
      if constexpr (STAGED<TPR, CH>) {
        ld16_async(mine + i * TPR * 16, there ? a.x + (long long)row * a.x_ld + c * 8 : a.x, there);
        if (a.residual) ld16_async(mine + (CH + i) * TPR * 16, there ? a.residual + (long long)row * a.residual_ld + c * 8 : a.residual, there);
      } else {
        v[i] = r[i] = make_uint4(0, 0, 0, 0);
        if (there) {
          v[i] = ld16(a.x + (long long)row * a.x_ld + c * 8);
          if (a.residual) r[i] = ld16(a.residual + (long long)row * a.residual_ld + c * 8);
        }
      }
    }
  };
  auto weights = [&](uint32_t c, f2 (&g)[4], f2 (&b)[4]) {
#pragma unroll
    for (int u = 0; u < 4; u += 2) {
      ulonglong2 w = make_ulonglong2(f2_pack(1.f, 1.f), f2_pack(1.f, 1.f)), z = make_ulonglong2(0, 0);
      if (c < pieces && a.gain) w = __ldg(reinterpret_cast<const ulonglong2*>(a.gain + c * 8 + 2 * u));
      if (c < pieces && a.bias) z = __ldg(reinterpret_cast<const ulonglong2*>(a.bias + c * 8 + 2 * u));
      g[u] = w.x; g[u + 1] = w.y;
      b[u] = z.x; b[u + 1] = z.y;
    }
  };
  const uint32_t step = gridDim.x * ROWS;
  uint32_t row = blockIdx.x * ROWS + threadIdx.x / TPR;
  fetch(row);
  f2 gain[KEEP ? CH : 1][4], bias[KEEP ? CH : 1][4];
  if constexpr (KEEP) {
#pragma unroll
    for (int i = 0; i < CH; ++i) weights(me + (uint32_t)i * TPR, gain[i], bias[i]);
  }
  for (uint32_t first = blockIdx.x * ROWS; first < rows; first += step, row += step) {
    const bool ok = row < rows;
    f2 h[CH][4];
    if constexpr (STAGED<TPR, CH>) ld16_async_wait();
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      if constexpr (STAGED<TPR, CH>) {
        v[0] = lds16(mine + i * TPR * 16);
        r[0] = a.residual ? lds16(mine + (CH + i) * TPR * 16) : make_uint4(0, 0, 0, 0);
      }
      const uint4 &x = v[STAGED<TPR, CH> ? 0 : i], &z = r[STAGED<TPR, CH> ? 0 : i];
      const uint32_t w[4] = {x.x, x.y, x.z, x.w}, e[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
      for (int u = 0; u < 4; ++u) h[i][u] = a.residual ? f2_add(bf16_2(w[u]), bf16_2(e[u])) : bf16_2(w[u]);
    }
    // the next row is on its way while this one goes through its reductions
    if (first + step < rows) fetch(row + step);
    if (a.total) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const uint32_t c = me + (uint32_t)i * TPR;
        if (c < pieces && ok) st_stream16(a.total + (long long)row * a.total_ld + c * 8, to_bf16x8(h[i]));
      }
    }
    if constexpr (KIND != NORM_NONE) {
      if constexpr (KIND == NORM_LAYER) {
        f2 s = 0;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
          for (int u = 0; u < 4; ++u) s = f2_add(s, h[i][u]);
        const float mu = row_sum<TPR>(f2_lo(s) + f2_hi(s), slot0) * per;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          if (me + (uint32_t)i * TPR < pieces) {
#pragma unroll
            for (int u = 0; u < 4; ++u) h[i][u] = f2_add(h[i][u], f2_pack(-mu, -mu));
          }
        }
      }
      f2 s = 0;
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int u = 0; u < 4; ++u) s = f2_fma(h[i][u], h[i][u], s);
      const float rstd = 1.0f / sqrtf(row_sum<TPR>(f2_lo(s) + f2_hi(s), slot1) * per + a.eps);
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        f2 g[4], b[4];
        if constexpr (!KEEP) weights(me + (uint32_t)i * TPR, g, b);
#pragma unroll
        for (int u = 0; u < 4; ++u)                    // (beyond the last column: zero before, zero with its bias of zero)
          h[i][u] = f2_fma(f2_mul(h[i][u], f2_pack(rstd, rstd)), KEEP ? gain[KEEP ? i : 0][u] : g[u], KEEP ? bias[KEEP ? i : 0][u] : b[u]);
      }
    }
    if (a.out) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const uint32_t c = me + (uint32_t)i * TPR;
        if (c < pieces && ok) st_stream16(a.out + (long long)row * a.out_ld + c * 8, to_bf16x8(h[i]));
      }
    }
    if (a.q) {
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int u = 0; u < 4; ++u) top = max_nan(top, h[i][u]);
      // magnitudes compare as integers: infinities are above all numbers, and NaN above them
      const uint32_t m = row_max<TPR>(__float_as_uint(top), slot2);
      top = __uint_as_float(m);
      const float scale = m >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : top < NORM_TINY ? 0.f : top / (a.format == LLMCACHE_I8 ? 127.f : 448.f);
      const float inv = 1.0f / scale;
      if (me == 0 && ok) a.scale[row] = scale;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const uint32_t c = me + (uint32_t)i * TPR;
        if (c < pieces && ok) {
          uint2 e = make_uint2(0, 0);
          if (scale > 0.f)
            e = a.format == LLMCACHE_I8 ? to_int8(h[i], f2_pack(inv, inv), f2_pack(-scale, -scale)) : to_e4m3(h[i], f2_pack(inv, inv), f2_pack(-scale, -scale));
          *reinterpret_cast<uint2*>(a.q + (long long)row * a.q_ld + c * 8) = e;
        }
      }
    }
    // rows with a single reduction: its slot may be written again only when all have read it
    if (TPR > 32 && (KIND == NORM_NONE || (KIND == NORM_RMS && !a.q))) __syncthreads();
  }
  if constexpr (STAGED<TPR, CH>) ld16_async_wait();      // (a block without a row: nothing of it is on its way when the block ends)
}

template <int TPR, uint32_t CH>
constexpr uint32_t stage_bytes(bool residual) { return STAGED<TPR, CH> ? Shape<TPR>::THREADS * CH * 16 * (residual ? 2 : 1) : 0; }
// blocks per SM that run at a time, without and with a residual, on each device that has been set up
template <int TPR, uint32_t CH, int KIND>
int g_resident[MAX_DEVICES][2];

template <int TPR, uint32_t CH, int KIND>
cudaError_t launch_shape(const NormArgs& a, int dev, int sm_count, cudaStream_t st) {
  constexpr uint32_t ROWS = Shape<TPR>::ROWS;
  const bool res = a.residual != nullptr;
  int per_sm = g_resident<TPR, CH, KIND>[dev][res];
  if (!per_sm) return cudaErrorInvalidDevice;           // (not set up)
  // As many blocks as run at a time: a second, partial wave of them would leave SMs idle.  With three large arrays or more besides q, reads and
  // writes of fewer rows at a time are easier on the memory (1,024 columns, residual and total: 124 us per 105 M elements with 12 blocks per SM, 114
  // with 10; with x and q alone 76 and 80).
  if (1 + (a.residual != nullptr) + (a.total != nullptr) + (a.out != nullptr) >= 3) per_sm -= per_sm / 6;
  const unsigned long long cap = (unsigned long long)sm_count * per_sm;
  unsigned long long blocks = ((unsigned long long)a.n_rows + ROWS - 1) / ROWS;
  if (blocks > cap) blocks = cap;
  return launch_k(k_norm<TPR, CH, KIND>, dim3((uint32_t)blocks), dim3(Shape<TPR>::THREADS), stage_bytes<TPR, CH>(res), st, a);
}

template <int TPR, int KIND, uint32_t CH = LEAST_CH<TPR>>
cudaError_t launch_width(const NormArgs& a, uint32_t ch, int dev, int sm_count, cudaStream_t st) {
  if (ch == CH) return launch_shape<TPR, CH, KIND>(a, dev, sm_count, st);
  if constexpr (CH < MOST_CH<TPR>) return launch_width<TPR, KIND, CH + 1>(a, ch, dev, sm_count, st);
  return cudaErrorInvalidValue;
}

// the same shapes, set up on the current device
template <int TPR, int KIND, uint32_t CH = LEAST_CH<TPR>>
cudaError_t setup_width(int dev) {
  cudaError_t e = cudaFuncSetAttribute(k_norm<TPR, CH, KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize, stage_bytes<TPR, CH>(true));
  for (int res = 0; res < 2 && e == cudaSuccess; ++res) {
    int per_sm = 0;
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, k_norm<TPR, CH, KIND>, Shape<TPR>::THREADS, stage_bytes<TPR, CH>(res != 0));
    if (e == cudaSuccess && per_sm < 1) e = cudaErrorInvalidConfiguration;
    if (e == cudaSuccess) g_resident<TPR, CH, KIND>[dev][res] = per_sm;
  }
  if constexpr (CH < MOST_CH<TPR>) return e == cudaSuccess ? setup_width<TPR, KIND, CH + 1>(dev) : e;
  return e;
}
template <int KIND>
cudaError_t setup_kind(int dev) {
  cudaError_t e = setup_width<8, KIND>(dev);
  if (e == cudaSuccess) e = setup_width<16, KIND>(dev);
  if (e == cudaSuccess) e = setup_width<32, KIND>(dev);
  if (e == cudaSuccess) e = setup_width<64, KIND>(dev);
  if (e == cudaSuccess) e = setup_width<128, KIND>(dev);
  if (e == cudaSuccess) e = setup_width<256, KIND>(dev);
  return e == cudaSuccess ? setup_width<512, KIND>(dev) : e;
}

template <int KIND>
cudaError_t launch_kind(const NormArgs& a, int dev, int sm_count, cudaStream_t st) {
  // As few threads without a piece of eight elements as there may be, with up to four pieces per thread (5,000 columns: 256 threads of three
  // pieces 104 us where 512 of two take 149); three per thread of a warp, whose registers hold the gains of no more (1,024 columns: 64
  // threads of two 113 us, 32 of four 121).  Up to eight for 256 threads,
  // with the next row in shared memory: 2,988 x 9,272, rms and total to e4m3 31 us, with 512 threads and the next row in registers 41; 4,000 x 12,288 49 and 59; 512 threads
  // only where there is an SM for every row (8 rows of 12,680: 4.0 us, 4.2 with 256).
  const uint32_t pieces = a.cols / 8, widest = a.n_rows <= (uint32_t)sm_count ? 512 : 256;
  uint32_t best = widest, least = ~0u;
  for (uint32_t threads = 8; threads <= widest; threads *= 2) {
    const uint32_t ch = (pieces + threads - 1) / threads, idle = threads * ch - pieces;
    // (MOST_CH; 256 threads take five and more only where 512 are not to be had)
    if (ch <= (threads <= 32 ? 3 : threads < widest || widest == 512 ? 4 : 8) && idle < least) { best = threads; least = idle; }
  }
  const uint32_t ch = (pieces + best - 1) / best;
  switch (best) {
    case 8: return launch_width<8, KIND>(a, ch, dev, sm_count, st);
    case 16: return launch_width<16, KIND>(a, ch, dev, sm_count, st);
    case 32: return launch_width<32, KIND>(a, ch, dev, sm_count, st);
    case 64: return launch_width<64, KIND>(a, ch, dev, sm_count, st);
    case 128: return launch_width<128, KIND>(a, ch, dev, sm_count, st);
    case 256: return launch_width<256, KIND>(a, ch, dev, sm_count, st);
    default: return launch_width<512, KIND>(a, ch, dev, sm_count, st);
  }
}

}  // namespace

cudaError_t setup_norm() {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev < 0 || dev >= MAX_DEVICES)) e = cudaErrorInvalidDevice;
  if (e == cudaSuccess) e = setup_kind<NORM_NONE>(dev);
  if (e == cudaSuccess) e = setup_kind<NORM_LAYER>(dev);
  return e == cudaSuccess ? setup_kind<NORM_RMS>(dev) : e;
}

cudaError_t launch_norm(const NormArgs& a, int sm_count, cudaStream_t st) {
  if (a.n_rows == 0) return cudaSuccess;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return cudaErrorInvalidDevice;
  switch (a.kind) {
    case NORM_NONE: return launch_kind<NORM_NONE>(a, dev, sm_count, st);
    case NORM_LAYER: return launch_kind<NORM_LAYER>(a, dev, sm_count, st);
    case NORM_RMS: return launch_kind<NORM_RMS>(a, dev, sm_count, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace llmc
