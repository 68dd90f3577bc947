// Received weights of a paged call, one thread per key.
#include "attn.cuh"
#include "ptx.cuh"

namespace llmc {

namespace {

// softmax exponent of a score in base-2 units; apart: key position - query position
__device__ __forceinline__ float modified(const ScoreArgs& m, float dot, uint32_t h, int32_t apart) {
  float z = dot * m.scale;
  if (m.cap > 0.f) z = m.cap * tanhf(z / m.cap);
  if (m.slopes) z -= m.slopes[h] * (float)abs(apart);
  if (m.table) z += m.table[(size_t)h * (2 * m.reach + 1) + min(max(apart, -m.reach), m.reach) + m.reach];
  return z;
}

__device__ __forceinline__ float dot64(const __nv_bfloat16* a, const float* b) {
  float s = 0.f;
  const uint4* p = reinterpret_cast<const uint4*>(a);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint4 w = p[i];
    const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      s = fmaf(__uint_as_float(q[u] << 16), b[i * 8 + 2 * u], s);
      s = fmaf(__uint_as_float(q[u] & 0xFFFF0000u), b[i * 8 + 2 * u + 1], s);
    }
  }
  return s;
}

// one thread per (sequence, key/value head, slot)
__global__ void __launch_bounds__(128) k_attn_weights_rows(AttnArgs a, uint32_t cap) {
  griddep_sync();
  const unsigned long long total = (unsigned long long)a.n_seqs * a.kv_heads * cap;
  for (unsigned long long id = (unsigned long long)blockIdx.x * 128 + threadIdx.x; id < total; id += (unsigned long long)gridDim.x * 128) {
    const uint32_t j = id % cap, hk = (id / cap) % a.kv_heads, s = id / cap / a.kv_heads;
    const SeqGeo g = seq_geo(a, s);
    if (j >= g.len) continue;
    float sum = 0.f;
    const int32_t p = page_of(a, s, j);
    const size_t side = ((size_t)s * a.kv_heads + hk) * a.side_ld + j;
    if (p >= 0) {
      float kk[64];
      const __nv_bfloat16* krow = a.k_pages + page_row(a, p, hk, j);
      for (int c = 0; c < 64; ++c) kk[c] = __bfloat162float(krow[c]);
      const int32_t kpos = a.positions ? a.positions[side] : (int32_t)j;
      for (uint32_t i = 0; i < g.cnt; ++i) {
        const long long my_slot = (long long)g.slot0 + i;
        if (a.m.causal && (long long)j > my_slot) continue;
        const long long qpos = a.first ? (long long)a.first[s] + i : my_slot;
        for (uint32_t h = hk * a.group; h < (hk + 1) * a.group; ++h) {
          const __nv_bfloat16* q = a.q.ptr + (long long)(g.row0 + i) * a.q.tok + (long long)h * a.q.head;
          const float lse = a.lse[(size_t)(g.row0 + i) * a.heads + h];
          const float z = modified(a.m, dot64(q, kk), h, (int32_t)(kpos - qpos));
          if (lse != -INFINITY) sum += expf(z - lse);
        }
      }
    }
    a.weights[side] = a.decay == 0.f ? sum : a.decay * a.weights[side] + sum;
  }
}

}  // namespace

cudaError_t setup_attn_kernels() { return setup_attn_tc(); }

cudaError_t launch_attn(const AttnArgs& a, float* part, size_t part_units, int sm_count, cudaStream_t st) {
  return launch_attn_tc(a, part, part_units, sm_count, st);
}

cudaError_t launch_attn_weights(const AttnArgs& a, int sm_count, cudaStream_t st) {
  const unsigned long long cap = (unsigned long long)a.pages_ld << a.page_shift;
  const uint32_t c = cap < a.max_len ? (uint32_t)cap : a.max_len;
  const unsigned long long blocks = ((unsigned long long)a.n_seqs * a.kv_heads * c + 127) / 128, most = (unsigned long long)sm_count * 16;
  if (blocks == 0) return cudaSuccess;
  return launch_k(k_attn_weights_rows, dim3((uint32_t)(blocks < most ? blocks : most)), dim3(128), 0, st, a, c);
}

}  // namespace llmc
