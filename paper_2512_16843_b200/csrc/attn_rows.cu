// Attention with score modifiers, one warp per query row and head: the simplest form of every case.
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

__global__ void __launch_bounds__(128) k_attn_rows(AttnArgs a) {
  griddep_sync();
  __shared__ float qs[4][64];
  const uint32_t lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const bool paged = a.pages != nullptr;
  uint32_t n_seqs = a.n_seqs;
  if (a.n_seqs_dev) n_seqs = min(n_seqs, *a.n_seqs_dev);
  const unsigned long long total = (unsigned long long)n_seqs * a.n * a.heads;
  for (unsigned long long id = (unsigned long long)blockIdx.x * 4 + w; id < total; id += (unsigned long long)gridDim.x * 4) {
    const uint32_t h = id % a.heads, hk = h / a.group;
    const uint32_t i = (id / a.heads) % a.n, s = id / a.heads / a.n;
    SeqGeo g{0, a.n, a.n, 0};
    if (paged) { g = seq_geo(a, s); if (i >= g.cnt) continue; }
    const long long my_slot = (long long)g.slot0 + i;
    const long long qpos = paged && a.first ? (long long)a.first[s] + i : my_slot;
    const size_t row = paged ? (size_t)g.row0 + i : (size_t)i;
    const __nv_bfloat16* q = a.q.ptr + (paged ? 0 : (long long)s * a.q.seq) + (long long)row * a.q.tok + (long long)h * a.q.head;
    __syncwarp();
    qs[w][lane * 2] = __bfloat162float(q[lane * 2]);
    qs[w][lane * 2 + 1] = __bfloat162float(q[lane * 2 + 1]);
    __syncwarp();
    const int32_t qdoc = a.m.doc ? a.m.doc[(size_t)s * a.n + i] : 0;
    const int32_t pre = a.m.prefix ? a.m.prefix[s] : 0;
    float mx = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
    for (uint32_t j0 = 0; j0 < g.len; j0 += 32) {
      const uint32_t j = j0 + lane;
      bool see = j < g.len && (!a.m.causal || (long long)j <= my_slot || (int32_t)j < pre);
      if (see && a.m.doc) { const int32_t kd = a.m.doc[(size_t)s * a.n + j]; see = kd == qdoc && kd >= 0; }
      const __nv_bfloat16* vrow = nullptr;
      float z = -INFINITY;
      if (see) {
        const __nv_bfloat16* krow;
        if (paged) {
          const int32_t p = page_of(a, s, j);
          if (p < 0) see = false;
          const size_t off = see ? page_row(a, p, hk, j) : 0;
          krow = a.k_pages + off; vrow = a.v_pages + off;
        } else {
          krow = a.k.ptr + (long long)s * a.k.seq + (long long)j * a.k.tok + (long long)hk * a.k.head;
          vrow = a.v.ptr + (long long)s * a.v.seq + (long long)j * a.v.tok + (long long)hk * a.v.head;
        }
        if (see) {
          const int32_t kpos = paged && a.positions ? a.positions[((size_t)s * a.kv_heads + hk) * a.side_ld + j] : (int32_t)j;
          z = modified(a.m, dot64(krow, qs[w]), h, (int32_t)(kpos - qpos));
        }
      }
      float tm = z;
      for (int o = 16; o > 0; o >>= 1) { const float x = __shfl_xor_sync(0xFFFFFFFFu, tm, o); tm = (tm != tm || x != x) ? NAN : fmaxf(tm, x); }
      if (tm == -INFINITY) continue;
      const float mn = (mx != mx || tm != tm) ? NAN : fmaxf(mx, tm);
      const float corr = mx == -INFINITY ? 0.f : expf(mx - mn);
      const float p = see ? expf(z - mn) : 0.f;
      float ls = p;
      for (int o = 16; o > 0; o >>= 1) ls += __shfl_xor_sync(0xFFFFFFFFu, ls, o);
      l = l * corr + ls;
      o0 *= corr; o1 *= corr;
      mx = mn;
      const uint32_t seen = __ballot_sync(0xFFFFFFFFu, see);
      for (int t = 0; t < 32; ++t) {
        if (!((seen >> t) & 1u)) continue;
        const float pt = __shfl_sync(0xFFFFFFFFu, p, t);
        const unsigned long long vp = __shfl_sync(0xFFFFFFFFu, (unsigned long long)vrow, t);
        const uint32_t v2 = reinterpret_cast<const uint32_t*>(vp)[lane];
        o0 = fmaf(pt, __uint_as_float(v2 << 16), o0);
        o1 = fmaf(pt, __uint_as_float(v2 & 0xFFFF0000u), o1);
      }
    }
    const float inv = mx == -INFINITY ? 0.f : 1.f / l;
    __nv_bfloat16* o = a.out.ptr + (paged ? 0 : (long long)s * a.out.seq) + (long long)row * a.out.tok + (long long)h * a.out.head;
    const bool none = mx == -INFINITY;
    reinterpret_cast<__nv_bfloat162*>(o)[lane] = __floats2bfloat162_rn(none ? 0.f : o0 * inv, none ? 0.f : o1 * inv);
    if (a.lse && lane == 0) a.lse[(paged ? row : (size_t)s * a.n + i) * a.heads + h] = none ? -INFINITY : mx + logf(l);
    __syncwarp();
  }
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

cudaError_t setup_attn_kernels() { return cudaSuccess; }

cudaError_t launch_attn(const AttnArgs& a, int sm_count, cudaStream_t st) {
  const unsigned long long total = (unsigned long long)a.n_seqs * a.n * a.heads;
  unsigned long long blocks = (total + 3) / 4, most = (unsigned long long)sm_count * 16;
  if (total == 0) return cudaSuccess;
  return launch_k(k_attn_rows, dim3((uint32_t)(blocks < most ? blocks : most)), dim3(128), 0, st, a);
}

cudaError_t launch_attn_weights(const AttnArgs& a, int sm_count, cudaStream_t st) {
  const unsigned long long cap = (unsigned long long)a.pages_ld << a.page_shift;
  const uint32_t c = cap < a.max_len ? (uint32_t)cap : a.max_len;
  const unsigned long long blocks = ((unsigned long long)a.n_seqs * a.kv_heads * c + 127) / 128, most = (unsigned long long)sm_count * 16;
  if (blocks == 0) return cudaSuccess;
  return launch_k(k_attn_weights_rows, dim3((uint32_t)(blocks < most ? blocks : most)), dim3(128), 0, st, a, c);
}

}  // namespace llmc
