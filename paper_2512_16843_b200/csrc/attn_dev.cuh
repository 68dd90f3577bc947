// Device helpers that the attention kernels share.
#pragma once
#include <cuda.h>
#include "attn.cuh"
#include "ptx.cuh"

namespace llmc {

// bf16 rows of 64 columns (llmcache_rows), boxes of box_heads x box_toks rows, 128-byte swizzle, zero fill outside
bool make_tensor_map_rows(CUtensorMap* map, const RowsArgs& r, uint64_t heads, uint64_t toks, uint64_t seqs, uint32_t box_heads,
                          uint32_t box_toks);

namespace {

__device__ __forceinline__ float ex2f(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float lg2f(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// A table entry in base-2 units.  The type's lowest value, a mask in some programs, stays finite, and entries near it count as
// it; -inf is dealt with apart.
__device__ __forceinline__ float entry2(float b) { return (b < -2.3e38f ? -2.3e38f : b) * LOG2E_F; }
// natural logarithm of the sum l of exponentials that refer to the maximum m (base 2)
__device__ __forceinline__ float log_sum(float m, float l) {
  const float x = (m + lg2f(l)) * LN2_F;
  return x < -2.29e38f ? -3.402823466e38f : x;               // (nothing but entries that count as the lowest value)
}
__device__ __forceinline__ float max3f(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// the loads before it are complete and their registers may be read (they pass through the statement)
__device__ __forceinline__ void tc_wait_ld32(uint32_t (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                 "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
               :: "memory");
  asm volatile("" : "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]),
                    "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31]) :: "memory");
}
__device__ __forceinline__ void tc_ld_16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
        "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tc_wait_ld16(uint32_t (&v)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                 "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
               :: "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive_n(uint32_t bar, uint32_t n) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(n) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0u;
}
// The loop of a wait, out of line: what is not ready at once has time for a call, and the code around stays together.
__device__ __noinline__ bool wait_long(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, unsigned long long limit_ns,
                                       uint32_t backoff_ns) {
  return mbar_wait(bar, parity, abort_flag, limit_ns, backoff_ns);
}
__device__ __forceinline__ bool wait_one(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, unsigned long long limit_ns) {
  return mbar_try(bar, parity) || wait_long(bar, parity, abort_flag, limit_ns, 0);
}
// mbar_wait by a whole warp: all lanes get the same answer, so that they leave together when a wait runs out
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, unsigned long long limit_ns,
                                          uint32_t backoff_ns) {
  if (__all_sync(0xFFFFFFFFu, mbar_try(bar, parity))) return true;
  return __all_sync(0xFFFFFFFFu, wait_long(bar, parity, abort_flag, limit_ns, backoff_ns));
}
__device__ __forceinline__ unsigned long long f2_dup(float x) { return f2_pack(x, x); }

// tanh of two values: an odd polynomial on |u| <= 0.75 (tanh_fit.py, relative error 1.4e-7)
__device__ __forceinline__ unsigned long long tanh_small2(unsigned long long u) {
  const unsigned long long s = f2_mul(u, u);
  unsigned long long q = f2_fma(f2_dup(-4.723952152e-03f), s, f2_dup(1.959378645e-02f));
  q = f2_fma(q, s, f2_dup(-5.334981903e-02f));
  q = f2_fma(q, s, f2_dup(1.332551539e-01f));
  q = f2_fma(q, s, f2_dup(-3.333296776e-01f));
  q = f2_fma(q, s, f2_dup(1.0f));
  return f2_mul(u, q);
}
// The same on |u| <= 0.4, with two terms less (2.1e-7).
__device__ __forceinline__ unsigned long long tanh_tiny2(unsigned long long u) {
  const unsigned long long s = f2_mul(u, u);
  unsigned long long q = f2_fma(f2_dup(-4.756107554e-02f), s, f2_dup(1.327115595e-01f));
  q = f2_fma(q, s, f2_dup(-3.333137333e-01f));
  q = f2_fma(q, s, f2_dup(9.999998808e-01f));
  return f2_mul(u, q);
}
constexpr float TANH_TINY = 0.4f, TANH_SMALL = 0.75f;        // largest arguments of the two
// 1 - 2 / (1 + e^2u): for |u| > 0.75, where the difference loses nothing
__device__ __forceinline__ float tanh_large(float u) { return 1.f - __fdividef(2.f, 1.f + ex2f(2.f * LOG2E_F * u)); }
// tanh of any two values.  Which form a value takes depends on the value alone: where a whole group of scores is small a kernel
// may call tanh_tiny2 for all of it, and no bit depends on what else the group holds (keys that a row does not see, rows that
// do not exist).
__device__ __forceinline__ unsigned long long tanh_any2(unsigned long long u) {
  const unsigned long long a = tanh_tiny2(u), b = tanh_small2(u);
  const float x = f2_lo(u), y = f2_hi(u), p = fabsf(x) <= TANH_TINY ? f2_lo(a) : f2_lo(b), q = fabsf(y) <= TANH_TINY ? f2_hi(a) : f2_hi(b);
  return f2_pack(fabsf(x) <= TANH_SMALL ? p : tanh_large(x), fabsf(y) <= TANH_SMALL ? q : tanh_large(y));
}

}  // namespace
}  // namespace llmc
