// C ABI of the miss-path transformer layer and of the layer-wise caching loop (Algorithm 1).
#include <cstdio>
#include <cstring>
#include <new>
#include "layer.cuh"
#include "attn_host.cuh"
#include "dense8.cuh"
#include "kv_rotate.cuh"
#include "ptx.cuh"

using namespace llmc;

struct llmcache_layer {
  llmcache_layer_desc desc{};
  int sm_count = 0;
  char* ws = nullptr;            // workspace
  bool owns_ws = false;
  __nv_bfloat16 *qkv = nullptr, *a = nullptr, *t = nullptr, *y = nullptr, *f = nullptr, *vt = nullptr;
  uint32_t* status = nullptr;    // device word: a bounded wait expired
  bool has_mods = false;         // llmcache_layer_score_mods
  ScoreArgs mods{};
  bool rms = false;              // llmcache_layer_rms
  RotateArgs rotate{nullptr, 0u, 0u};            // llmcache_layer_rotation; dims 0: none
  uint32_t format = LLMCACHE_BF16;               // of the products (llmcache_layer_quantise)
  char* ws8 = nullptr;                           // 8-bit weights and their scales
  bool owns_ws8 = false;
  const uint8_t* w8[4] = {};                     // q|k|v, o, 1, 2
  const float* s8[4] = {};
};

namespace llmc {
bool layer_masks_by_sequence(const llmcache_layer* L) { return L && L->has_mods && (L->mods.doc || L->mods.prefix); }
}

namespace {
constexpr size_t WS_ALIGN = 256;
inline size_t up256(size_t x) { return (x + WS_ALIGN - 1) / WS_ALIGN * WS_ALIGN; }

int check_layer_desc(const llmcache_layer_desc* d) {
  if (!d || d->struct_size != sizeof(llmcache_layer_desc)) return LLMCACHE_ERR_ARG;
  if (d->d_model == 0 || d->heads == 0 || d->ffn == 0 || d->seq_len == 0 || d->max_seqs == 0) return LLMCACHE_ERR_SHAPE;
  if (d->d_model % 64 != 0 || d->ffn % 64 != 0) return LLMCACHE_ERR_SHAPE;
  if (d->d_model != d->heads * 64) return LLMCACHE_ERR_UNSUPPORTED;       // head size 64 only
  if ((unsigned long long)d->max_seqs * d->seq_len > 0xFFFFFFFFull) return LLMCACHE_ERR_SHAPE;
  const void* ptrs[] = {d->w_qkv, d->b_qkv, d->w_o, d->b_o, d->ln1_g, d->ln1_b, d->w_1, d->b_1, d->w_2, d->b_2,
                        d->ln2_g, d->ln2_b};
  for (const void* p : ptrs)
    if (!p || ((uintptr_t)p & 15u)) return LLMCACHE_ERR_ARG;
  if (d->workspace && ((uintptr_t)d->workspace % WS_ALIGN)) return LLMCACHE_ERR_ARG;
  return LLMCACHE_OK;
}

size_t layer_ws_bytes(const llmcache_layer_desc& d) {
  const size_t T = (size_t)d.max_seqs * d.seq_len;
  const size_t vt = (size_t)d.max_seqs * d.d_model * attention_vt_pitch(d.seq_len) * 2;      // per-head transposes of V
  return up256(T * 3 * d.d_model * 2) + 3 * up256(T * d.d_model * 2) + up256(T * d.ffn * 2) + up256(vt) + WS_ALIGN;
}

// attention over the sequences of one forward call: q|k|v rows of 3d columns in, rows of d columns out
AttnArgs layer_attn_args(const llmcache_layer* L, uint32_t n_seqs, const uint32_t* n_seqs_dev) {
  const long long d = L->desc.d_model, n = L->desc.seq_len;
  AttnArgs a{};
  a.q = RowsArgs{L->qkv, n * 3 * d, 3 * d, 64};
  a.k = RowsArgs{L->qkv + d, n * 3 * d, 3 * d, 64};
  a.v = RowsArgs{L->qkv + 2 * d, n * 3 * d, 3 * d, 64};
  a.out = RowsArgs{L->a, n * d, d, 64};
  a.heads = a.kv_heads = L->desc.heads;
  a.group = 1;
  a.n_seqs = n_seqs;
  a.n_seqs_dev = n_seqs_dev;
  a.n = L->desc.seq_len;
  a.m = L->mods;
  a.status = L->status;
  return a;
}

enum { P_QKV = 0, P_O = 1, P_1 = 2, P_2 = 3 };                   // the layer's products
struct Eight { uint8_t* q; float* scale; long long ld; };       // rows in 8 bits

// The norms and products of one forward or extend call, in the layer's number format.  After an error nothing more is launched.
struct LayerSteps {
  const llmcache_layer* L;
  uint32_t rows;
  const uint32_t* count;         // rows = min(rows, *count * per)
  uint32_t per;
  cudaStream_t st;
  cudaError_t e = cudaSuccess;

  bool in8() const { return L->format != LLMCACHE_BF16; }
  // rows of d bytes and their scales in the memory of a [rows, d] bf16 matrix: d >= 64, so the scales fit behind them
  Eight eight_in(__nv_bfloat16* m) const {
    const size_t most = (size_t)L->desc.max_seqs * L->desc.seq_len * L->desc.d_model;
    return Eight{(uint8_t*)m, (float*)((char*)m + most), (long long)L->desc.d_model};
  }
  // rows of f in 8 bits: each in the first half of its own place (the kernel reads a row before it writes it); the scales
  // where the q|k|v rows were
  Eight eight_f() const { return Eight{(uint8_t*)L->f, (float*)L->qkv, 2ll * L->desc.ffn}; }

  void run_norm(uint32_t kind, const __nv_bfloat16* x, uint32_t cols, const float* g, const float* b, __nv_bfloat16* y, const Eight* q) {
    if (e != cudaSuccess) return;
    NormArgs a{};
    a.x = x; a.out = y; a.gain = g; a.bias = b;
    a.x_ld = a.out_ld = cols;
    if (q) { a.q = q->q; a.scale = q->scale; a.q_ld = q->ld; a.format = L->format; }
    a.n_rows = rows; a.cols = cols; a.kind = kind; a.eps = L->desc.eps;
    a.count_dev = count; a.rows_per_count = per;
    e = launch_norm(a, L->sm_count, st);
  }
  // the layer's norm of x: y in bf16, q in 8 bits (either may be null)
  void norm(const __nv_bfloat16* x, const float* g, const float* b, __nv_bfloat16* y, const Eight* q) {
    if (e != cudaSuccess) return;
    if (L->rms || q) run_norm(L->rms ? NORM_RMS : NORM_LAYER, x, L->desc.d_model, g, b, y, q);
    else e = launch_layernorm(x, g, b, y, rows, L->desc.d_model, count, per, L->desc.eps, L->sm_count, st);
  }
  void to8(const __nv_bfloat16* x, uint32_t cols, const Eight& q) { run_norm(NORM_NONE, x, cols, nullptr, nullptr, nullptr, &q); }
  // product `which` of x (8-bit layers: of q)
  void product(int which, const __nv_bfloat16* x, const Eight& q, const void* w, const float* bias, const __nv_bfloat16* res,
               __nv_bfloat16* o, uint32_t N, uint32_t K, uint32_t act, VtOut vt = VtOut{nullptr, 0, 0, 0}) {
    if (e != cudaSuccess) return;
    if (!in8()) {
      e = launch_gemm(x, (const __nv_bfloat16*)w, bias, res, o, L->status, rows, N, K, count, per, act, L->sm_count, st, vt);
      return;
    }
    DenseArgs a{};
    a.a = q.q; a.a_scale = q.scale; a.a_ld = q.ld;
    a.w = L->w8[which]; a.w_scale = L->s8[which]; a.w_ld = K;
    a.bias = bias; a.residual = res; a.residual_ld = N; a.out = o; a.out_ld = N;
    a.m = rows; a.n = N; a.k = K; a.act = act; a.format = L->format;
    a.count_dev = count; a.rows_per_count = per;
    a.status = L->status;
    a.vt = vt;
    e = launch_dense8(a, L->sm_count, st);
  }

  // from the layer's input to q|k|v
  void before_attention(const __nv_bfloat16* X, VtOut vt) {
    const llmcache_layer_desc& D = L->desc;
    const Eight y8 = eight_in(L->y);
    if (D.pre_ln) norm(X, D.ln1_g, D.ln1_b, in8() ? nullptr : L->y, in8() ? &y8 : nullptr);
    else if (in8()) to8(X, D.d_model, y8);
    product(P_QKV, D.pre_ln ? L->y : X, y8, D.w_qkv, D.b_qkv, nullptr, L->qkv, 3 * D.d_model, D.d_model, LAYER_ACT_NONE, vt);
  }
  // from the attention's output to the layer's
  void behind_attention(const __nv_bfloat16* X, __nv_bfloat16* O) {
    const llmcache_layer_desc& D = L->desc;
    const uint32_t d = D.d_model, act = D.tanh_gelu ? LAYER_ACT_GELU_TANH : LAYER_ACT_GELU_ERF;
    const Eight y8 = eight_in(L->y), a8 = eight_in(L->a), f8 = eight_f();
    if (in8()) to8(L->a, d, y8);
    product(P_O, L->a, y8, D.w_o, D.b_o, X, L->t, d, d, LAYER_ACT_NONE);
    // post-norm: y is the next residual too, so its 8 bits go where the attention's output was
    norm(L->t, D.pre_ln ? D.ln2_g : D.ln1_g, D.pre_ln ? D.ln2_b : D.ln1_b, in8() && D.pre_ln ? nullptr : L->y, in8() ? &a8 : nullptr);
    product(P_1, L->y, a8, D.w_1, D.b_1, nullptr, L->f, D.ffn, d, act);
    if (in8()) to8(L->f, D.ffn, f8);
    product(P_2, L->f, f8, D.w_2, D.b_2, D.pre_ln ? L->t : L->y, D.pre_ln ? O : L->t, d, D.ffn, LAYER_ACT_NONE);
    if (!D.pre_ln) norm(L->t, D.ln2_g, D.ln2_b, O, nullptr);
  }
};

// sizes of the weight matrices: rows (output channels) and columns
void weight_shape(const llmcache_layer_desc& D, int which, uint32_t* rows, uint32_t* cols) {
  const uint32_t d = D.d_model;
  *rows = which == P_QKV ? 3 * d : which == P_1 ? D.ffn : d;
  *cols = which == P_2 ? D.ffn : d;
}
size_t layer_ws8_bytes(const llmcache_layer_desc& D) {
  size_t total = 0;
  for (int w = 0; w < 4; ++w) {
    uint32_t r, c;
    weight_shape(D, w, &r, &c);
    total += up256((size_t)r * c) + up256((size_t)r * 4);
  }
  return total;
}
constexpr uint32_t NORM_MOST = 16384;      // columns of a row that k_norm takes
// whether k_norm can stand in for the layer's norms (its rows are counted in 31 bits)
bool norm_serves(const llmcache_layer_desc& D) {
  return D.d_model <= NORM_MOST && (uint64_t)D.max_seqs * D.seq_len <= 0x7FFFFFFFull;
}
}  // namespace

extern "C" {

int llmcache_layer_bytes(const llmcache_layer_desc* desc, size_t* bytes_out) {
  if (!bytes_out) return LLMCACHE_ERR_ARG;
  int rc = check_layer_desc(desc);
  if (rc != LLMCACHE_OK) return rc;
  *bytes_out = layer_ws_bytes(*desc);
  return LLMCACHE_OK;
}

int llmcache_layer_create(const llmcache_layer_desc* desc, llmcache_layer_t** layer_out) {
  if (!layer_out) return LLMCACHE_ERR_ARG;
  *layer_out = nullptr;
  int rc = check_layer_desc(desc);
  if (rc != LLMCACHE_OK) return rc;
  int ndev = 0;
  if (cudaGetDeviceCount(&ndev) != cudaSuccess || ndev <= 0) { cudaGetLastError(); return LLMCACHE_ERR_CUDA; }
  if (desc->device < 0 || desc->device >= ndev) return LLMCACHE_ERR_ARG;
  int prev = 0;
  cudaGetDevice(&prev);
  if (cudaSetDevice(desc->device) != cudaSuccess) { cudaGetLastError(); return LLMCACHE_ERR_CUDA; }
  llmcache_layer* L = new (std::nothrow) llmcache_layer();
  if (!L) { cudaSetDevice(prev); return LLMCACHE_ERR_NOMEM; }
  L->desc = *desc;
  if (L->desc.eps <= 0.f) L->desc.eps = 1e-5f;
  const size_t need = layer_ws_bytes(*desc);
  cudaError_t e = cudaDeviceGetAttribute(&L->sm_count, cudaDevAttrMultiProcessorCount, desc->device);
  if (e == cudaSuccess) {
    if (desc->workspace) {
      if (desc->workspace_bytes < need) { delete L; cudaSetDevice(prev); return LLMCACHE_ERR_NOMEM; }
      L->ws = (char*)desc->workspace;
    } else {
      if (cudaMalloc((void**)&L->ws, need) != cudaSuccess) { cudaGetLastError(); delete L; cudaSetDevice(prev); return LLMCACHE_ERR_NOMEM; }
      L->owns_ws = true;
    }
  }
  if (e == cudaSuccess) {
    const size_t T = (size_t)desc->max_seqs * desc->seq_len, d = desc->d_model;
    char* p = L->ws;
    L->status = (uint32_t*)p; p += WS_ALIGN;
    L->qkv = (__nv_bfloat16*)p; p += up256(T * 3 * d * 2);
    L->a = (__nv_bfloat16*)p; p += up256(T * d * 2);
    L->t = (__nv_bfloat16*)p; p += up256(T * d * 2);
    L->y = (__nv_bfloat16*)p; p += up256(T * d * 2);
    L->f = (__nv_bfloat16*)p; p += up256(T * desc->ffn * 2);
    L->vt = (__nv_bfloat16*)p;
    e = cudaMemset(L->status, 0, WS_ALIGN);
  }
  if (e == cudaSuccess) e = setup_gemm_kernel();
  if (e == cudaSuccess) e = setup_attention_kernel();
  if (e == cudaSuccess) e = setup_attn_kernels();
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  cudaSetDevice(prev);
  if (e != cudaSuccess) {
    cudaGetLastError();
    if (L->owns_ws) cudaFree(L->ws);
    delete L;
    return LLMCACHE_ERR_CUDA;
  }
  *layer_out = L;
  return LLMCACHE_OK;
}

int llmcache_layer_destroy(llmcache_layer_t* L) {
  if (!L) return LLMCACHE_ERR_ARG;
  int prev = 0;
  cudaGetDevice(&prev);
  cudaSetDevice(L->desc.device);
  cudaError_t e = cudaDeviceSynchronize();
  if (L->owns_ws) cudaFree(L->ws);
  if (L->owns_ws8) cudaFree(L->ws8);
  cudaSetDevice(prev);
  delete L;
  return e == cudaSuccess ? LLMCACHE_OK : LLMCACHE_ERR_CUDA;
}

int llmcache_layer_forward(llmcache_layer_t* L, const void* x, uint32_t n_seqs, const uint32_t* n_seqs_dev,
                           void* out, void* stream) {
  if (!L || (n_seqs && (!x || !out))) return LLMCACHE_ERR_ARG;
  if (n_seqs > L->desc.max_seqs) return LLMCACHE_ERR_SHAPE;
  if (((uintptr_t)x | (uintptr_t)out) & 15u) return LLMCACHE_ERR_ARG;
  if (n_seqs == 0) return LLMCACHE_OK;
  if (L->has_mods && L->mods.mask_seqs && n_seqs > L->mods.mask_seqs) return LLMCACHE_ERR_SHAPE;
  int prev = 0;
  cudaGetDevice(&prev);
  if (prev != L->desc.device && cudaSetDevice(L->desc.device) != cudaSuccess) { cudaGetLastError(); return LLMCACHE_ERR_CUDA; }
  const llmcache_layer_desc& D = L->desc;
  const uint32_t n = D.seq_len, d = D.d_model, T = n_seqs * n;
  cudaStream_t st = (cudaStream_t)stream;
  const __nv_bfloat16* X = (const __nv_bfloat16*)x;
  LayerSteps steps{L, T, n_seqs_dev, n, st};
  cudaError_t& e = steps.e;
  // the V third of the q|k|v product is written transposed per head (what the attention kernel reads); the kernel with
  // score modifiers reads all of q|k|v from the one matrix
  steps.before_attention(X, L->has_mods ? VtOut{nullptr, 0, 0, 0} : VtOut{L->vt, 2 * d, attention_vt_pitch(n), D.heads});
  if (e == cudaSuccess && L->rotate.dims) {
    AttnArgs r = layer_attn_args(L, n_seqs, n_seqs_dev);
    r.out = r.q;
    r.n_rows = T;
    r.q.seq = r.k.seq = r.out.seq = 0;                     // (rows are numbered through)
    e = launch_kv_rotate(r, L->rotate, L->sm_count, st);
  }
  if (e == cudaSuccess)
    e = L->has_mods ? launch_attn(layer_attn_args(L, n_seqs, n_seqs_dev), AttnScratch{}, L->sm_count, st)
                    : launch_attention_tc(L->qkv, L->vt, L->a, L->status, n, d, D.heads, n_seqs, n_seqs_dev, D.causal, st);
  steps.behind_attention(X, (__nv_bfloat16*)out);
  if (prev != L->desc.device) cudaSetDevice(prev);
  if (e != cudaSuccess) { cudaGetLastError(); return LLMCACHE_ERR_CUDA; }
  return LLMCACHE_OK;
}

int llmcache_layer_score_mods(llmcache_layer_t* L, const llmcache_score_mods* mods) {
  if (!L) return LLMCACHE_ERR_ARG;
  if (!mods) { L->has_mods = false; return LLMCACHE_OK; }
  ScoreArgs m;
  const int rc = check_score_mods(mods, &m);
  if (rc != LLMCACHE_OK) return rc;
  if ((m.causal != 0) != (L->desc.causal != 0)) return LLMCACHE_ERR_ARG;
  for (const void* p : {(const void*)m.slopes, (const void*)m.table, (const void*)m.doc, (const void*)m.prefix})
    if (p && !pointer_on_device(p, L->desc.device)) return LLMCACHE_ERR_ARG;
  L->mods = m;
  L->has_mods = true;
  return LLMCACHE_OK;
}

int llmcache_layer_rms(llmcache_layer_t* L, uint32_t on) {
  if (!L || on > 1) return LLMCACHE_ERR_ARG;
  if (on && !norm_serves(L->desc)) return LLMCACHE_ERR_UNSUPPORTED;
  if (on) {
    int prev = 0;
    cudaGetDevice(&prev);
    if (prev != L->desc.device && cudaSetDevice(L->desc.device) != cudaSuccess) { cudaGetLastError(); return LLMCACHE_ERR_CUDA; }
    const cudaError_t e = setup_eight();
    if (prev != L->desc.device) cudaSetDevice(prev);
    if (e != cudaSuccess) { cudaGetLastError(); return LLMCACHE_ERR_CUDA; }
  }
  L->rms = on != 0;
  return LLMCACHE_OK;
}

int llmcache_layer_rotation(llmcache_layer_t* L, const llmcache_rotation* rotation) {
  if (!L) return LLMCACHE_ERR_ARG;
  RotateArgs r;
  const int rc = check_rotation(rotation, &r);
  if (rc != LLMCACHE_OK) return rc;
  if (r.dims && !pointer_on_device(r.inv_freq, L->desc.device)) return LLMCACHE_ERR_ARG;
  L->rotate = r;
  return LLMCACHE_OK;
}

int llmcache_layer_quantise_bytes(llmcache_layer_t* L, size_t* bytes_out) {
  if (!L || !bytes_out) return LLMCACHE_ERR_ARG;
  *bytes_out = layer_ws8_bytes(L->desc);
  return LLMCACHE_OK;
}

int llmcache_layer_quantise(llmcache_layer_t* L, uint32_t format, void* workspace, size_t workspace_bytes, void* stream) {
  if (!L) return LLMCACHE_ERR_ARG;
  if (format != LLMCACHE_BF16 && format != LLMCACHE_I8 && format != LLMCACHE_E4M3) return LLMCACHE_ERR_ARG;
  const llmcache_layer_desc& D = L->desc;
  const size_t need = layer_ws8_bytes(D);
  if (format != LLMCACHE_BF16) {
    if (!norm_serves(D) || D.ffn > NORM_MOST) return LLMCACHE_ERR_UNSUPPORTED;
    if ((uintptr_t)workspace % WS_ALIGN) return LLMCACHE_ERR_ARG;
    if (workspace && workspace_bytes < need) return LLMCACHE_ERR_NOMEM;
    if (workspace && !pointer_on_device(workspace, D.device)) return LLMCACHE_ERR_ARG;
  }
  int prev = 0;
  cudaGetDevice(&prev);
  if (prev != D.device && cudaSetDevice(D.device) != cudaSuccess) { cudaGetLastError(); return LLMCACHE_ERR_CUDA; }
  const bool eight = format != LLMCACHE_BF16, was_eight = L->format != LLMCACHE_BF16;
  cudaError_t e = eight ? setup_eight() : cudaSuccess;
  int rc = LLMCACHE_OK;
  // The new weights' memory before anything of the layer changes: the caller's, the library's that is there already (its size depends on
  // the layer alone), or new.
  char* to = (char*)workspace;
  bool fresh = false;
  if (eight && !workspace) {
    to = L->owns_ws8 ? L->ws8 : nullptr;
    if (!to && e == cudaSuccess) {
      fresh = cudaMalloc((void**)&to, need) == cudaSuccess;
      if (!fresh) { cudaGetLastError(); rc = LLMCACHE_ERR_NOMEM; }
    }
  }
  if (e == cudaSuccess && rc == LLMCACHE_OK && was_eight) e = cudaDeviceSynchronize();      // calls in flight still read the weights that are there
  if (e == cudaSuccess && rc == LLMCACHE_OK && eight) {
    if (was_eight && to < L->ws8 + need && L->ws8 < to + need) L->format = LLMCACHE_BF16;   // (the old weights go while the new ones come)
    const void* from[4] = {D.w_qkv, D.w_o, D.w_1, D.w_2};
    const uint8_t* w8[4];
    const float* s8[4];
    char* at = to;
    for (int w = 0; w < 4 && e == cudaSuccess; ++w) {
      uint32_t r, c;
      weight_shape(D, w, &r, &c);
      NormArgs a{};
      a.x = (const __nv_bfloat16*)from[w]; a.x_ld = c;
      a.q = (uint8_t*)at; a.q_ld = c; at += up256((size_t)r * c);
      a.scale = (float*)at; at += up256((size_t)r * 4);
      a.n_rows = r; a.cols = c; a.kind = NORM_NONE; a.format = format; a.rows_per_count = 1;
      e = launch_norm(a, L->sm_count, (cudaStream_t)stream);
      w8[w] = a.q;
      s8[w] = a.scale;
    }
    if (e == cudaSuccess) {
      if (L->owns_ws8 && to != L->ws8) cudaFree(L->ws8);
      L->ws8 = to;
      L->owns_ws8 = !workspace;
      L->format = format;
      for (int w = 0; w < 4; ++w) { L->w8[w] = w8[w]; L->s8[w] = s8[w]; }
    }
  }
  if (e != cudaSuccess && fresh) {
    cudaDeviceSynchronize();
    cudaFree(to);
  }
  if (e == cudaSuccess && !eight && was_eight) {
    if (L->owns_ws8) cudaFree(L->ws8);
    L->ws8 = nullptr;
    L->owns_ws8 = false;
    L->format = LLMCACHE_BF16;
  }
  if (prev != D.device) cudaSetDevice(prev);
  if (e != cudaSuccess) { cudaGetLastError(); return LLMCACHE_ERR_CUDA; }
  return rc;
}

int llmcache_layer_extend(llmcache_layer_t* L, llmcache_kv_t* kv, const void* x, const llmcache_kv_chunk* chunk,
                          void* out, void* stream) {
  if (!L || !kv || !chunk || chunk->struct_size != sizeof(llmcache_kv_chunk)) return LLMCACHE_ERR_ARG;
  const llmcache_layer_desc& D = L->desc;
  if (!D.causal || layer_masks_by_sequence(L)) return LLMCACHE_ERR_UNSUPPORTED;
  int rc = kv_fits_layer(kv, D.device, D.heads);
  if (rc != LLMCACHE_OK) return rc;
  const uint32_t T = chunk->n_rows, d = D.d_model;
  if ((uint64_t)T > (uint64_t)D.max_seqs * D.seq_len) return LLMCACHE_ERR_SHAPE;
  if (T && chunk->n_seqs && (!x || !out || !chunk->cu_rows)) return LLMCACHE_ERR_ARG;
  if (((uintptr_t)x | (uintptr_t)out) & 15u) return LLMCACHE_ERR_ARG;
  // the attention's arguments: q, k and v are the thirds of the rows that the first product writes
  llmcache_score_mods m{};
  m.struct_size = sizeof(m);
  m.causal = 1;
  if (L->has_mods) { m.scale = L->mods.scale; m.cap = L->mods.cap; m.reach = (uint32_t)L->mods.reach; m.slopes = L->mods.slopes; m.table = L->mods.table; }
  llmcache_kv_chunk c = *chunk;
  c.q = llmcache_rows{L->qkv, 0, 3ll * d, 64};
  c.k_new = llmcache_rows{L->qkv + d, 0, 3ll * d, 64};
  c.v_new = llmcache_rows{L->qkv + 2 * d, 0, 3ll * d, 64};
  c.out = llmcache_rows{L->a, 0, (int64_t)d, 64};
  c.mods = &m;
  llmcache_kv_new nw{};                                    // rotated rows go into the cache ahead of the attention
  if (L->rotate.dims) {
    nw.struct_size = sizeof(nw);
    nw.n_seqs = c.n_seqs; nw.n_rows = c.n_rows; nw.pages_ld = c.pages_ld;
    nw.cu_rows = c.cu_rows; nw.lens = c.lens; nw.pages = c.pages;
    nw.k_new = c.k_new; nw.v_new = c.v_new; nw.q = nw.q_out = c.q;
    nw.positions = c.positions; nw.first = c.first; nw.side_ld = c.side_ld;
    c.k_new = c.v_new = llmcache_rows{nullptr, 0, 0, 0};
    if (!c.positions) c.first = nullptr;                   // (without positions only the rotation asks for it)
  }
  rc = kv_check_chunk(kv, &c);
  if (rc == LLMCACHE_OK && L->rotate.dims) rc = kv_check_append(kv, &nw);
  if (rc != LLMCACHE_OK || T == 0 || c.n_seqs == 0) return rc;

  int prev = 0;
  cudaGetDevice(&prev);
  if (prev != D.device && cudaSetDevice(D.device) != cudaSuccess) { cudaGetLastError(); return LLMCACHE_ERR_CUDA; }
  cudaStream_t st = (cudaStream_t)stream;
  const __nv_bfloat16* X = (const __nv_bfloat16*)x;
  // rows behind the last sequence are neither computed nor written
  LayerSteps steps{L, T, (const uint32_t*)(c.cu_rows + c.n_seqs), 1, st};
  cudaError_t& e = steps.e;
  steps.before_attention(X, VtOut{nullptr, 0, 0, 0});
  if (e == cudaSuccess && L->rotate.dims) rc = kv_append(kv, &nw, &L->rotate, st);
  if (e == cudaSuccess && rc == LLMCACHE_OK) rc = kv_attend(kv, &c, true, st);
  if (rc == LLMCACHE_OK) steps.behind_attention(X, (__nv_bfloat16*)out);
  if (prev != D.device) cudaSetDevice(prev);
  if (e != cudaSuccess) { cudaGetLastError(); return LLMCACHE_ERR_CUDA; }
  return rc;
}

int llmcache_layer_status(llmcache_layer_t* L) {
  if (!L) return LLMCACHE_ERR_ARG;
  uint32_t s = 0;
  if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&s, L->status, 4, cudaMemcpyDeviceToHost) != cudaSuccess) {
    cudaGetLastError();
    return LLMCACHE_ERR_CUDA;
  }
  return s ? LLMCACHE_ERR_TIMEOUT : LLMCACHE_OK;
}

int llmcache_layer_debug_knobs(llmcache_layer_t* L, uint64_t wait_limit_ns, uint32_t flags) {
  if (!L) return LLMCACHE_ERR_ARG;
  uint32_t w[3] = {flags, (uint32_t)(wait_limit_ns & 0xFFFFFFFFull), (uint32_t)(wait_limit_ns >> 32)};
  if (cudaDeviceSynchronize() != cudaSuccess ||
      cudaMemcpy(L->status + 1, w, sizeof(w), cudaMemcpyHostToDevice) != cudaSuccess) {
    cudaGetLastError();
    return LLMCACHE_ERR_CUDA;
  }
  return LLMCACHE_OK;
}

// Algorithm 1 with fingerprint-on-write: only layer 1 pools its input; every later probe takes the position means
// that the previous layer's row movers produced.  pooled == nullptr: each bank's own buffer carries them.
static int infer_fused(llmcache_bank_t** banks, llmcache_layer_t** layers, uint32_t n_layers, const void* h0,
                       uint32_t B, float tau, void* buf_a, void* buf_b, void* h_miss, void* miss_out,
                       llmcache_probe_io* io, float* pooled, void** h_final, void* stream) {
  const void* cur = h0;
  void* bufs[2] = {buf_a, buf_b};
  const float* prev_means = nullptr;
  int rc = LLMCACHE_OK;
  for (uint32_t l = 0; l < n_layers && rc == LLMCACHE_OK; ++l) {
    void* next = bufs[l & 1u];
    const uint32_t ld = banks[l]->desc.d_model;
    float* means_out = pooled ? pooled : banks[l]->a.pooled_own;
    io->h_miss = h_miss;
    // the rows this layer writes are summed on the way: means_out then holds the next layer's position means.
    // (With one shared buffer the probe has consumed its previous contents before the commit overwrites them.)
    rc = llmcache_bank_pool_out(banks[l], l + 1 < n_layers ? means_out : nullptr, ld);
    if (rc != LLMCACHE_OK) break;
    if (l == 0) rc = llmcache_probe(banks[l], cur, B, tau, next, io, stream);
    else        rc = llmcache_probe_pooled(banks[l], prev_means, ld, cur, B, tau, next, io, stream);
    if (rc == LLMCACHE_OK) rc = llmcache_layer_forward(layers[l], h_miss, B, io->counts + 1, miss_out, stream);
    if (rc == LLMCACHE_OK) rc = llmcache_commit(banks[l], miss_out, io, next, nullptr, stream);
    if (rc == LLMCACHE_OK) rc = llmcache_bank_pool_out(banks[l], nullptr, 0);
    prev_means = means_out;
    cur = next;
  }
  if (rc != LLMCACHE_OK) return rc;
  *h_final = const_cast<void*>(cur);
  return LLMCACHE_OK;
}

int llmcache_infer(llmcache_bank_t** banks, llmcache_layer_t** layers, uint32_t n_layers, const void* h0, uint32_t B,
                   float tau, void* buf_a, void* buf_b, void* h_miss, void* miss_out, llmcache_probe_io* io,
                   void** h_final, void* stream) {
  if (!layers || !h0 || !buf_a || !buf_b || !h_final || n_layers == 0) return LLMCACHE_ERR_ARG;
  if (banks && (!io || !h_miss || !miss_out)) return LLMCACHE_ERR_ARG;
  // masks of single sequences: the misses change their places, and a match does not look at masks
  for (uint32_t l = 0; banks && l < n_layers; ++l)
    if (layer_masks_by_sequence(layers[l])) return LLMCACHE_ERR_UNSUPPORTED;
  if (banks) {
    // banks created with fused_pool (all of them, same width) take the fingerprint-on-write path by themselves
    bool fused = true;
    for (uint32_t l = 0; l < n_layers; ++l)
      fused = fused && banks[l] && banks[l]->a.pooled_own && banks[l]->desc.d_model == banks[0]->desc.d_model &&
              B <= banks[l]->desc.max_batch;
    if (fused) return infer_fused(banks, layers, n_layers, h0, B, tau, buf_a, buf_b, h_miss, miss_out, io, nullptr,
                                  h_final, stream);
  }
  const void* cur = h0;
  void* bufs[2] = {buf_a, buf_b};
  for (uint32_t l = 0; l < n_layers; ++l) {
    void* next = bufs[l & 1u];
    int rc;
    if (banks) {
      // Algorithm 1: lookup (hits take the stored output), layer on the compacted misses, insert
      io->h_miss = h_miss;
      rc = llmcache_probe(banks[l], cur, B, tau, next, io, stream);
      if (rc == LLMCACHE_OK) rc = llmcache_layer_forward(layers[l], h_miss, B, io->counts + 1, miss_out, stream);
      if (rc == LLMCACHE_OK) rc = llmcache_commit(banks[l], miss_out, io, next, nullptr, stream);
    } else {
      rc = llmcache_layer_forward(layers[l], cur, B, nullptr, next, stream);    // no caching: every layer in full
    }
    if (rc != LLMCACHE_OK) return rc;
    cur = next;
  }
  *h_final = const_cast<void*>(cur);
  return LLMCACHE_OK;
}

int llmcache_infer_pooled(llmcache_bank_t** banks, llmcache_layer_t** layers, uint32_t n_layers, const void* h0,
                          uint32_t B, float tau, void* buf_a, void* buf_b, void* h_miss, void* miss_out,
                          llmcache_probe_io* io, float* pooled, void** h_final, void* stream) {
  if (!banks || !layers || !h0 || !buf_a || !buf_b || !h_final || n_layers == 0) return LLMCACHE_ERR_ARG;
  if (!io || !h_miss || !miss_out || !pooled) return LLMCACHE_ERR_ARG;
  for (uint32_t l = 0; l < n_layers; ++l)
    if (layer_masks_by_sequence(layers[l])) return LLMCACHE_ERR_UNSUPPORTED;
  return infer_fused(banks, layers, n_layers, h0, B, tau, buf_a, buf_b, h_miss, miss_out, io, pooled, h_final, stream);
}

}  // extern "C"
