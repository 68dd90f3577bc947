// C ABI of the attention operators: llmcache_attention and the paged key/value cache (llmcache_kv_*).
#include <algorithm>
#include <cstring>
#include <mutex>
#include <new>
#include "attn.cuh"
#include "attn_host.cuh"
#include "ptx.cuh"

using namespace llmc;

namespace {

constexpr size_t WS_ALIGN = 256;
inline size_t up256(size_t x) { return (x + WS_ALIGN - 1) / WS_ALIGN * WS_ALIGN; }
inline bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// Makes `device` current for the scope; false if that fails.
struct OnDevice {
  int prev = -1, dev;
  bool ok;
  explicit OnDevice(int d) : dev(d) {
    ok = cudaGetDevice(&prev) == cudaSuccess && (prev == dev || cudaSetDevice(dev) == cudaSuccess);
    if (!ok) cudaGetLastError();
  }
  ~OnDevice() { if (ok && prev != dev) cudaSetDevice(prev); }
};

int done(cudaError_t e) {
  if (e == cudaSuccess) return LLMCACHE_OK;
  cudaGetLastError();
  return LLMCACHE_ERR_CUDA;
}

int read_status(const uint32_t* status) {
  uint32_t s = 0;
  if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&s, status, 4, cudaMemcpyDeviceToHost) != cudaSuccess) {
    cudaGetLastError();
    return LLMCACHE_ERR_CUDA;
  }
  return s ? LLMCACHE_ERR_TIMEOUT : LLMCACHE_OK;
}

int write_knobs(uint32_t* status, uint64_t wait_limit_ns, uint32_t flags) {
  const uint32_t w[3] = {flags, (uint32_t)(wait_limit_ns & 0xFFFFFFFFull), (uint32_t)(wait_limit_ns >> 32)};
  if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(status + 1, w, sizeof(w), cudaMemcpyHostToDevice) != cudaSuccess) {
    cudaGetLastError();
    return LLMCACHE_ERR_CUDA;
  }
  return LLMCACHE_OK;
}

// strides of a row array; dimensions of size one need none
int take_rows(const llmcache_rows* r, uint64_t seqs, uint64_t toks, uint64_t heads, RowsArgs* o) {
  if (!r || !r->ptr || !aligned(r->ptr, 16)) return LLMCACHE_ERR_ARG;
  const int64_t st[3] = {r->seq_stride, r->tok_stride, r->head_stride};
  const uint64_t dim[3] = {seqs, toks, heads};
  long long out[3];
  for (int i = 0; i < 3; ++i) {
    if (dim[i] <= 1) { out[i] = 0; continue; }
    if (st[i] <= 0 || st[i] % 8 != 0 || st[i] > (1ll << 38)) return LLMCACHE_ERR_ARG;
    out[i] = st[i];
  }
  *o = RowsArgs{(__nv_bfloat16*)r->ptr, out[0], out[1], out[2]};
  return LLMCACHE_OK;
}

// ---- llmcache_attention without an object: status words per device, looked up once --------------------------
__device__ __align__(16) uint32_t g_attn_status[4];
constexpr int MAX_DEVICES = 64;
struct Dev { bool ready = false; uint32_t* status = nullptr; int sm_count = 0; };
Dev g_dev[MAX_DEVICES];
std::mutex g_mu;

cudaError_t device_setup(int dev, Dev* out) {
  std::lock_guard<std::mutex> lock(g_mu);
  Dev& d = g_dev[dev];
  if (!d.ready) {
    uint32_t* p = nullptr;
    cudaError_t e = cudaGetSymbolAddress((void**)&p, g_attn_status);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&d.sm_count, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = setup_attn_kernels();
    if (e != cudaSuccess) return e;
    d.status = p;
    d.ready = true;
  }
  *out = d;
  return cudaSuccess;
}

int current_device(int* dev) {
  if (cudaGetDevice(dev) == cudaSuccess && *dev >= 0 && *dev < MAX_DEVICES) return LLMCACHE_OK;
  cudaGetLastError();
  return LLMCACHE_ERR_CUDA;
}

}  // namespace

namespace llmc {

int check_score_mods(const llmcache_score_mods* m, ScoreArgs* o) {
  *o = ScoreArgs{0.125f, 0.f, 0u, 0, nullptr, nullptr, nullptr, nullptr, 0u};
  if (!m) return LLMCACHE_OK;
  if (m->struct_size != sizeof(llmcache_score_mods)) return LLMCACHE_ERR_ARG;
  if (!(m->scale >= 0.f) || m->scale > 1e30f) return LLMCACHE_ERR_ARG;
  if (m->cap != 0.f && !(m->cap >= 1e-3f && m->cap <= 1e30f)) return LLMCACHE_ERR_ARG;
  if (m->causal > 1) return LLMCACHE_ERR_ARG;
  if (m->table && m->reach > 1024) return LLMCACHE_ERR_SHAPE;
  if (!aligned(m->slopes, 4) || !aligned(m->table, 4) || !aligned(m->doc, 4) || !aligned(m->prefix, 4)) return LLMCACHE_ERR_ARG;
  if (m->prefix && !m->causal) return LLMCACHE_ERR_ARG;
  o->scale = m->scale == 0.f ? 0.125f : m->scale;
  o->cap = m->cap;
  o->causal = m->causal;
  o->reach = (int32_t)m->reach;
  o->slopes = m->slopes; o->table = m->table; o->doc = m->doc; o->prefix = m->prefix;
  o->mask_seqs = m->doc || m->prefix ? m->mask_seqs : 0u;
  return LLMCACHE_OK;
}

int kv_fits_layer(const llmcache_kv* kv, int device, uint32_t heads) {
  if (kv->desc.device != device) return LLMCACHE_ERR_ARG;
  return kv->desc.heads == heads && kv->desc.kv_heads == heads ? LLMCACHE_OK : LLMCACHE_ERR_SHAPE;
}

}  // namespace llmc

namespace {

int check_kv_desc(const llmcache_kv_desc* d) {
  if (!d || d->struct_size != sizeof(llmcache_kv_desc)) return LLMCACHE_ERR_ARG;
  if (!d->k_pages || !d->v_pages || !aligned(d->k_pages, 16) || !aligned(d->v_pages, 16)) return LLMCACHE_ERR_ARG;
  if (!aligned(d->workspace, WS_ALIGN)) return LLMCACHE_ERR_ARG;
  if (!d->heads || !d->kv_heads || d->heads % d->kv_heads || d->heads > 65536) return LLMCACHE_ERR_SHAPE;
  if (d->heads / d->kv_heads > ATTN_MAX_GROUP) return LLMCACHE_ERR_UNSUPPORTED;
  if (!d->num_pages || !d->max_seqs || !d->max_rows || !d->max_len) return LLMCACHE_ERR_SHAPE;
  if (d->page_size < 16 || d->page_size > 256 || (d->page_size & (d->page_size - 1))) return LLMCACHE_ERR_SHAPE;
  if (d->num_pages > 0x7FFFFFFFu || d->max_len > (1u << 30) || d->max_seqs > (1u << 20) || d->max_rows > (1u << 28)) return LLMCACHE_ERR_SHAPE;
  const uint64_t dense = (uint64_t)d->kv_heads * d->page_size * 64;
  if (d->page_stride && (d->page_stride % 64 || d->page_stride < dense)) return LLMCACHE_ERR_SHAPE;
  // rows of 64 elements are addressed with signed 32-bit coordinates
  if ((d->page_stride ? d->page_stride : dense) / 64 * d->num_pages > 0x7FFFFFFFull) return LLMCACHE_ERR_SHAPE;
  return LLMCACHE_OK;
}

// (row, head, share of the keys) results of one call: a fixed budget of 22 MB, and a limit of the shares.  Where a call's rows
// and heads leave room for fewer shares than the launch would like, it takes as many as fit (250 and 166 rows of 16 heads: 12,
// where three items per SM would be 13).
constexpr size_t KV_PART_UNITS = 2 * 256 * 160;
// Scores of few rows are kept for the weights where they fit: 4 bytes per row and key, up to 64 MB.  (A call that needs more
// has its scores formed again from the keys.)
constexpr size_t KV_SCORE_FLOATS = 16u << 20;
size_t kv_score_floats(const llmcache_kv_desc& d) {
  // a token for every sequence, its tiles filled up
  const size_t most = (size_t)d.max_seqs * d.heads * (((size_t)d.max_len + 127) / 128 * 128);
  return most < KV_SCORE_FLOATS ? most : KV_SCORE_FLOATS;
}
struct KvLayout { size_t status, arrived, part, scores, stat, kept, count, total; };
KvLayout kv_layout(const llmcache_kv_desc& d) {
  KvLayout L{};
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o += up256(bytes); return at; };
  L.status = take(16);
  L.arrived = take((size_t)d.max_seqs * d.kv_heads * 4);
  L.part = take(KV_PART_UNITS * PART_FLOATS * 4);
  L.scores = take(kv_score_floats(d) * 4);
  L.stat = take((size_t)d.max_rows * d.heads * 8);
  L.kept = take((size_t)d.max_seqs * d.kv_heads * d.max_len * 4);
  L.count = take((size_t)d.max_seqs * 4);
  L.total = o;
  return L;
}

uint32_t log2_of(uint32_t x) { uint32_t s = 0; while ((1u << s) < x) ++s; return s; }

// What a call may name of each sequence's slots.
int check_side(const llmcache_kv* kv, uint32_t n_seqs, uint32_t pages_ld, const void* lens, const void* pages,
               bool has_side, uint64_t side_ld) {
  if (n_seqs > kv->desc.max_seqs) return LLMCACHE_ERR_SHAPE;
  if (!lens || !pages || !aligned(lens, 4) || !aligned(pages, 4)) return LLMCACHE_ERR_ARG;
  if (pages_ld == 0 || pages_ld > (1u << 30)) return LLMCACHE_ERR_SHAPE;
  const uint64_t most = (uint64_t)pages_ld * kv->desc.page_size;
  if (has_side && side_ld < (most < kv->desc.max_len ? most : kv->desc.max_len)) return LLMCACHE_ERR_SHAPE;
  return LLMCACHE_OK;
}

// Checks one call and fills in the kernels' arguments; o->n_seqs == 0: nothing to do.
int chunk_args(const llmcache_kv* kv, const llmcache_kv_chunk* c, AttnArgs* o) {
  if (!kv || !c || c->struct_size != sizeof(llmcache_kv_chunk)) return LLMCACHE_ERR_ARG;
  const llmcache_kv_desc& D = kv->desc;
  AttnArgs& a = *o;
  int rc = check_score_mods(c->mods, &a.m);
  if (rc != LLMCACHE_OK) return rc;
  if (a.m.doc || a.m.prefix) return LLMCACHE_ERR_UNSUPPORTED;
  if (!c->mods) a.m.causal = 1;
  if (c->n_rows > D.max_rows || c->longest > c->n_rows) return LLMCACHE_ERR_SHAPE;
  if (c->n_seqs > D.max_seqs) return LLMCACHE_ERR_SHAPE;
  if (c->n_seqs == 0 || c->n_rows == 0) return LLMCACHE_OK;
  if ((rc = check_side(kv, c->n_seqs, c->pages_ld, c->lens, c->pages, c->weights || c->positions, c->side_ld)) != LLMCACHE_OK) return rc;
  if (!c->cu_rows || !aligned(c->cu_rows, 4) || !aligned(c->lse, 4) || !aligned(c->weights, 4) || !aligned(c->positions, 4) ||
      !aligned(c->first, 4))
    return LLMCACHE_ERR_ARG;
  if (c->first && !c->positions) return LLMCACHE_ERR_ARG;
  if (c->weights && !(c->decay >= 0.f && c->decay <= 1.f)) return LLMCACHE_ERR_ARG;
  if ((rc = take_rows(&c->q, 1, c->n_rows, D.heads, &a.q)) != LLMCACHE_OK) return rc;
  if ((rc = take_rows(&c->out, 1, c->n_rows, D.heads, &a.out)) != LLMCACHE_OK) return rc;
  if ((c->k_new.ptr == nullptr) != (c->v_new.ptr == nullptr)) return LLMCACHE_ERR_ARG;
  if (c->k_new.ptr) {
    if ((rc = take_rows(&c->k_new, 1, c->n_rows, D.kv_heads, &a.k)) != LLMCACHE_OK) return rc;
    if ((rc = take_rows(&c->v_new, 1, c->n_rows, D.kv_heads, &a.v)) != LLMCACHE_OK) return rc;
  }
  a.lse = c->lse;
  a.stat = c->weights ? kv->stat : nullptr;
  a.heads = D.heads; a.kv_heads = D.kv_heads; a.group = D.heads / D.kv_heads;
  a.n_seqs = c->n_seqs; a.n = c->longest ? c->longest : c->n_rows;
  a.status = kv->status;
  a.cu = c->cu_rows; a.lens = c->lens; a.pages = c->pages; a.first = c->first;
  a.positions = c->positions; a.weights = c->weights; a.decay = c->decay;
  a.n_rows = c->n_rows; a.pages_ld = c->pages_ld; a.num_pages = D.num_pages; a.page_shift = log2_of(D.page_size);
  a.max_len = D.max_len; a.side_ld = c->side_ld; a.page_stride = D.page_stride;
  a.k_pages = (__nv_bfloat16*)D.k_pages; a.v_pages = (__nv_bfloat16*)D.v_pages;
  return LLMCACHE_OK;
}

}  // namespace

namespace llmc {
int kv_check_chunk(const llmcache_kv* kv, const llmcache_kv_chunk* c) {
  AttnArgs a{};
  return chunk_args(kv, c, &a);
}

int kv_attend(llmcache_kv* kv, const llmcache_kv_chunk* c, bool zero_rest, cudaStream_t st) {
  AttnArgs a{};
  int rc = chunk_args(kv, c, &a);
  if (rc != LLMCACHE_OK || a.n_seqs == 0) return rc;
  a.zero_rest = zero_rest && a.n < a.n_rows;
  if (a.weights && attn_is_few(a)) {
    const uint64_t cap = std::min<uint64_t>(a.max_len, (uint64_t)a.pages_ld << a.page_shift), ld = (cap + 127) / 128 * 128;
    const uint64_t rows = (uint64_t)a.n * a.group;
    if ((uint64_t)a.n_seqs * a.kv_heads * rows * ld <= kv->score_floats) {
      a.scores = kv->scores;
      a.score_ld = (uint32_t)ld;
      a.score_rows = (uint32_t)rows;
    }
  }
  OnDevice on(kv->desc.device);
  if (!on.ok) return LLMCACHE_ERR_CUDA;
  if (!attn_is_few(a) && (a.k.ptr || a.positions || (a.weights && a.decay != 0.f))) {
    const cudaError_t e = launch_kv_append(a, kv->sm_count, st);
    if (e != cudaSuccess) return done(e);
  }
  rc = launch_attn_checked(a, AttnScratch{kv->part, KV_PART_UNITS, kv->arrived}, kv->sm_count, st);
  if (rc == LLMCACHE_OK && a.weights) rc = done(launch_attn_weights(a, kv->sm_count, st));
  return rc;
}
}  // namespace llmc

extern "C" {

int llmcache_attention(const llmcache_rows* q, const llmcache_rows* k, const llmcache_rows* v, const llmcache_rows* out,
                       uint32_t n_seqs, uint32_t seq_len, uint32_t heads, uint32_t kv_heads, const uint32_t* n_seqs_dev,
                       const llmcache_score_mods* mods, float* lse, void* stream) {
  AttnArgs a{};
  int rc = check_score_mods(mods, &a.m);
  if (rc != LLMCACHE_OK) return rc;
  if (heads && kv_heads && heads % kv_heads == 0 && heads / kv_heads > ATTN_MAX_GROUP) return LLMCACHE_ERR_UNSUPPORTED;
  if (!heads || !kv_heads || heads % kv_heads || heads > 65536 || !seq_len || seq_len > (1u << 30)) return LLMCACHE_ERR_SHAPE;
  if (n_seqs == 0) return LLMCACHE_OK;                     // an empty batch has no buffers to check
  if (a.m.mask_seqs && n_seqs > a.m.mask_seqs) return LLMCACHE_ERR_SHAPE;
  if ((rc = take_rows(q, n_seqs, seq_len, heads, &a.q)) != LLMCACHE_OK) return rc;
  if ((rc = take_rows(k, n_seqs, seq_len, kv_heads, &a.k)) != LLMCACHE_OK) return rc;
  if ((rc = take_rows(v, n_seqs, seq_len, kv_heads, &a.v)) != LLMCACHE_OK) return rc;
  if ((rc = take_rows(out, n_seqs, seq_len, heads, &a.out)) != LLMCACHE_OK) return rc;
  if (!aligned(lse, 4) || !aligned(n_seqs_dev, 4)) return LLMCACHE_ERR_ARG;
  int dev = -1;
  if ((rc = current_device(&dev)) != LLMCACHE_OK) return rc;
  Dev d;
  cudaError_t e = device_setup(dev, &d);
  if (e != cudaSuccess) return done(e);
  if (!pointer_on_device(q->ptr, dev)) return LLMCACHE_ERR_ARG;      // (a tensor of another GPU, or of the host, would fault)
  a.lse = lse;
  a.heads = heads; a.kv_heads = kv_heads; a.group = heads / kv_heads;
  a.n_seqs = n_seqs; a.n_seqs_dev = n_seqs_dev; a.n = seq_len;
  a.status = d.status;
  return launch_attn_checked(a, AttnScratch{}, d.sm_count, (cudaStream_t)stream);
}

int llmcache_attention_status(void) {
  int dev = -1;
  int rc = current_device(&dev);
  if (rc != LLMCACHE_OK) return rc;
  const uint32_t* status;
  {
    std::lock_guard<std::mutex> lock(g_mu);
    if (!g_dev[dev].ready) return LLMCACHE_OK;             // never used on this device
    status = g_dev[dev].status;
  }
  return read_status(status);
}

int llmcache_attention_debug_knobs(uint64_t wait_limit_ns, uint32_t flags) {
  int dev = -1;
  int rc = current_device(&dev);
  if (rc != LLMCACHE_OK) return rc;
  uint32_t* status;
  {
    std::lock_guard<std::mutex> lock(g_mu);
    if (!g_dev[dev].ready) return LLMCACHE_ERR_STATE;
    status = g_dev[dev].status;
  }
  return write_knobs(status, wait_limit_ns, flags);
}

int llmcache_kv_bytes(const llmcache_kv_desc* desc, size_t* bytes_out) {
  if (!bytes_out) return LLMCACHE_ERR_ARG;
  const int rc = check_kv_desc(desc);
  if (rc != LLMCACHE_OK) return rc;
  *bytes_out = kv_layout(*desc).total;
  return LLMCACHE_OK;
}

int llmcache_kv_create(const llmcache_kv_desc* desc, llmcache_kv_t** kv_out) {
  if (!kv_out) return LLMCACHE_ERR_ARG;
  *kv_out = nullptr;
  int rc = check_kv_desc(desc);
  if (rc != LLMCACHE_OK) return rc;
  const KvLayout lay = kv_layout(*desc);
  if (desc->workspace && desc->workspace_bytes < lay.total) return LLMCACHE_ERR_NOMEM;
  int ndev = 0;
  if (cudaGetDeviceCount(&ndev) != cudaSuccess || ndev <= 0) { cudaGetLastError(); return LLMCACHE_ERR_CUDA; }
  if (desc->device < 0 || desc->device >= ndev) return LLMCACHE_ERR_ARG;
  OnDevice on(desc->device);
  if (!on.ok) return LLMCACHE_ERR_CUDA;
  llmcache_kv* kv = new (std::nothrow) llmcache_kv();
  if (!kv) return LLMCACHE_ERR_NOMEM;
  kv->desc = *desc;
  if (!kv->desc.page_stride) kv->desc.page_stride = (uint64_t)desc->kv_heads * desc->page_size * 64;
  if (desc->workspace) {
    kv->ws = (char*)desc->workspace;
  } else {
    if (cudaMalloc((void**)&kv->ws, lay.total) != cudaSuccess) { cudaGetLastError(); delete kv; return LLMCACHE_ERR_NOMEM; }
    kv->owns_ws = true;
  }
  kv->status = (uint32_t*)(kv->ws + lay.status);
  kv->arrived = (uint32_t*)(kv->ws + lay.arrived);
  kv->part = (float*)(kv->ws + lay.part);
  kv->scores = (float*)(kv->ws + lay.scores);
  kv->score_floats = kv_score_floats(*desc);
  kv->stat = (float2*)(kv->ws + lay.stat);
  kv->kept = (int32_t*)(kv->ws + lay.kept);
  kv->count = (uint32_t*)(kv->ws + lay.count);
  cudaError_t e = cudaMemset(kv->status, 0, lay.part);     // status and arrival counts
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&kv->sm_count, cudaDevAttrMultiProcessorCount, desc->device);
  if (e == cudaSuccess) e = setup_attn_kernels();
  if (e == cudaSuccess && attn_few_part_floats(kv->sm_count) > KV_PART_UNITS * PART_FLOATS) e = cudaErrorInvalidConfiguration;
  if (e == cudaSuccess) e = setup_evict_kernels();
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) {
    cudaGetLastError();
    if (kv->owns_ws) cudaFree(kv->ws);
    delete kv;
    return LLMCACHE_ERR_CUDA;
  }
  *kv_out = kv;
  return LLMCACHE_OK;
}

int llmcache_kv_destroy(llmcache_kv_t* kv) {
  if (!kv) return LLMCACHE_ERR_ARG;
  OnDevice on(kv->desc.device);
  const cudaError_t e = cudaDeviceSynchronize();
  if (kv->owns_ws) cudaFree(kv->ws);
  delete kv;
  return done(e);
}

int llmcache_kv_attention(llmcache_kv_t* kv, const llmcache_kv_chunk* c, void* stream) {
  return kv_attend(kv, c, false, (cudaStream_t)stream);
}

int llmcache_kv_evict(llmcache_kv_t* kv, const llmcache_kv_eviction* v, void* stream) {
  if (!kv || !v || v->struct_size != sizeof(llmcache_kv_eviction)) return LLMCACHE_ERR_ARG;
  const llmcache_kv_desc& D = kv->desc;
  if (v->budget == 0 || v->budget > D.max_len || (uint64_t)v->recent + v->sinks > v->budget) return LLMCACHE_ERR_SHAPE;
  if (v->n_seqs > D.max_seqs) return LLMCACHE_ERR_SHAPE;
  if (v->n_seqs == 0) return LLMCACHE_OK;
  int rc = check_side(kv, v->n_seqs, v->pages_ld, v->lens, v->pages, true, v->side_ld);
  if (rc != LLMCACHE_OK) return rc;
  if (!v->new_pages || !v->new_lens || !v->weights) return LLMCACHE_ERR_ARG;
  const void* ptrs[] = {v->new_pages, v->new_lens, v->weights, v->positions, v->new_weights, v->new_positions, v->kept};
  for (const void* p : ptrs)
    if (!aligned(p, 4)) return LLMCACHE_ERR_ARG;
  if ((uint64_t)v->new_pages_ld * D.page_size < v->budget) return LLMCACHE_ERR_SHAPE;
  if ((v->new_weights || v->new_positions) && v->new_side_ld < v->budget) return LLMCACHE_ERR_SHAPE;
  const uint64_t blocks = (uint64_t)v->n_seqs * D.kv_heads * ((v->budget + 63) / 64);
  if (blocks > 0x7FFFFFFFull) return LLMCACHE_ERR_SHAPE;
  EvictArgs a{};
  a.n_seqs = v->n_seqs; a.kv_heads = D.kv_heads; a.budget = v->budget; a.recent = v->recent; a.sinks = v->sinks;
  a.pages_ld = v->pages_ld; a.new_pages_ld = v->new_pages_ld; a.num_pages = D.num_pages;
  a.page_shift = log2_of(D.page_size); a.max_len = D.max_len;
  a.side_ld = v->side_ld; a.new_side_ld = v->new_side_ld; a.page_stride = D.page_stride;
  a.lens = v->lens; a.pages = v->pages; a.new_pages = v->new_pages; a.new_lens = v->new_lens;
  a.weights = v->weights; a.positions = v->positions;
  a.new_weights = v->new_weights; a.new_positions = v->new_positions;
  a.kept_out = v->kept; a.kept = kv->kept; a.count = kv->count;
  a.k_pages = (__nv_bfloat16*)D.k_pages; a.v_pages = (__nv_bfloat16*)D.v_pages;
  OnDevice on(D.device);
  if (!on.ok) return LLMCACHE_ERR_CUDA;
  return done(launch_evict_tokens(a, kv->sm_count, (cudaStream_t)stream));
}

int llmcache_kv_status(llmcache_kv_t* kv) {
  if (!kv) return LLMCACHE_ERR_ARG;
  OnDevice on(kv->desc.device);
  return on.ok ? read_status(kv->status) : LLMCACHE_ERR_CUDA;
}

int llmcache_kv_debug_knobs(llmcache_kv_t* kv, uint64_t wait_limit_ns, uint32_t flags) {
  if (!kv) return LLMCACHE_ERR_ARG;
  OnDevice on(kv->desc.device);
  return on.ok ? write_knobs(kv->status, wait_limit_ns, flags) : LLMCACHE_ERR_CUDA;
}

}  // extern "C"
