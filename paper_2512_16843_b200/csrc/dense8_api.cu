// C ABI of the operators with 8-bit values: llmcache_norm and llmcache_dense.  Neither takes an object; status words and launch
// attributes are looked up once per device.
#include <mutex>
#include "dense8.cuh"
#include "ptx.cuh"

using namespace llmc;

namespace {

inline bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

__device__ __align__(16) uint32_t g_dense_status[4];
constexpr int MAX_DEVICES = 64;
struct Dev { bool ready = false; uint32_t* status = nullptr; int sm_count = 0; uint32_t form = 0; };      // form: llmcache_dense_debug_knobs
Dev g_dev[MAX_DEVICES];
std::mutex g_mu;

int done(cudaError_t e) {
  if (e == cudaSuccess) return LLMCACHE_OK;
  cudaGetLastError();
  return LLMCACHE_ERR_CUDA;
}

// The current device's entry, set up on first use.  All of the library's set-up of these kernels is here, behind one lock: launches read
// what it writes without the lock, each behind a call of this function.
cudaError_t ready(int* dev, Dev* out) {
  const cudaError_t at = cudaGetDevice(dev);
  if (at != cudaSuccess) return at;
  if (*dev < 0 || *dev >= MAX_DEVICES) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(g_mu);
  Dev& d = g_dev[*dev];
  if (!d.ready) {
    uint32_t* p = nullptr;
    cudaError_t e = cudaGetSymbolAddress((void**)&p, g_dense_status);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&d.sm_count, cudaDevAttrMultiProcessorCount, *dev);
    if (e == cudaSuccess) e = setup_dense8_tc();
    if (e == cudaSuccess) e = setup_dense8_few();
    if (e == cudaSuccess) e = setup_norm();
    if (e != cudaSuccess) return e;
    d.status = p;
    d.ready = true;
  }
  *out = d;
  return cudaSuccess;
}

// a matrix of `rows` rows: its leading dimension, a multiple of `step` and at least `cols` (of no account for a single row)
bool take_ld(int64_t ld, uint64_t rows, uint64_t cols, uint32_t step, long long* out) {
  if (rows <= 1) { *out = (long long)((cols + step - 1) / step * step); return true; }
  if (ld < (int64_t)cols || ld % step != 0 || ld > (1ll << 32)) return false;
  *out = ld;
  return true;
}

constexpr uint32_t MOST_ROWS = 0x7FFFFFFFu;

// whether a form that was asked for (llmcache_dense_debug_knobs) can serve a call; m is not zero
bool form_serves(const DenseArgs& a, uint32_t form) {
  if (form == LLMCACHE_DENSE_FEW) return a.m <= 32;
  if (form < LLMCACHE_DENSE_CLUSTERS_2) return true;
  const uint64_t parts = 2ull << (form - LLMCACHE_DENSE_CLUSTERS_2);
  return (a.k + 127) / 128 >= parts && ((uint64_t)a.m + 127) / 128 * (((uint64_t)a.n + 63) / 64) * parts <= 0x7FFFFFFFull;
}

}  // namespace

namespace llmc {

cudaError_t setup_eight() {
  int dev = -1;
  Dev d;
  return ready(&dev, &d);
}

// What k_dense8_few takes, in us: a launch, and the bytes of weights that the busiest SM has to read, at the rate at which its warps feed
// mma.sync with 8, 16 or 32 tokens.  (Measured at 64 x 512 to 50,257 x 768 and 8,192 x 8,192.)
static float few_time(const DenseArgs& a, int sm_count) {
  constexpr float FIXED[2][3] = {{1.8f, 2.3f, 2.7f}, {1.8f, 2.3f, 4.4f}};
  constexpr float PER_BYTE[2][3] = {{28e-6f, 38e-6f, 52e-6f}, {30e-6f, 55e-6f, 92e-6f}};        // int8, e4m3
  const int t = a.format == LLMCACHE_I8 ? 0 : 1, n = a.m <= 8 ? 0 : a.m <= 16 ? 1 : 2;
  const float one = 16.0f * a.k, all = (float)a.n * a.k / sm_count;
  return FIXED[t][n] + PER_BYTE[t][n] * (one > all ? one : all);
}

cudaError_t launch_dense8(const DenseArgs& a, int sm_count, cudaStream_t st) {
  if (a.m == 0) return cudaSuccess;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return cudaErrorInvalidDevice;
  // Up to 8 rows (16 of int8) the weights are all there is to read, and a stream of them through registers is never behind (1,024 x 4,096, 8 rows: 3.1 us, 6.6
  // the other way; 8,192 x 8,192, 16 rows of int8 17 and 17); up to 32 it depends on how many there are (32 rows of int8, 1,024 x 4,096: 5.7 and
  // 6.0; 4,096 x 1,024: 4.5 and 5.6; 8,192 x 8,192: 36 and 17; 50,257 x 768: 22 and 13).
  const uint32_t always = a.format == LLMCACHE_I8 ? 16 : 8;
  if (a.m <= always && !a.vt.ptr) return launch_dense8_few(a, sm_count, st);
  const DenseForm f = choose_dense8_tc(a, dev, sm_count);
  if (a.m <= 32 && !a.vt.ptr && few_time(a, sm_count) < f.us) return launch_dense8_few(a, sm_count, st);
  return launch_dense8_tc(a, f.form, dev, sm_count, st);
}

}  // namespace llmc

extern "C" {

int llmcache_norm(const llmcache_norm_args* n, void* stream) {
  if (!n || n->struct_size != sizeof(llmcache_norm_args)) return LLMCACHE_ERR_ARG;
  if (n->kind > LLMCACHE_NORM_RMS || !(n->eps == n->eps) || n->eps > 1e30f) return LLMCACHE_ERR_ARG;
  if (n->kind == LLMCACHE_NORM_NONE && (n->gain || n->bias)) return LLMCACHE_ERR_ARG;
  if ((n->q == nullptr) != (n->scale == nullptr)) return LLMCACHE_ERR_ARG;
  if (n->q && n->format != LLMCACHE_I8 && n->format != LLMCACHE_E4M3) return LLMCACHE_ERR_ARG;
  if (n->cols == 0 || n->cols % 8 || n->cols > 16384 || n->n_rows > MOST_ROWS) return LLMCACHE_ERR_SHAPE;
  if (n->n_rows == 0) return LLMCACHE_OK;
  if (!n->x || (!n->total && !n->out && !n->q)) return LLMCACHE_ERR_ARG;
  const void* wide[] = {n->x, n->residual, n->total, n->out, n->gain, n->bias};
  for (const void* p : wide)
    if (!aligned(p, 16)) return LLMCACHE_ERR_ARG;
  if (!aligned(n->q, 8) || !aligned(n->scale, 4) || !aligned(n->count_dev, 4)) return LLMCACHE_ERR_ARG;
  NormArgs a{};
  if (!take_ld(n->x_ld, n->n_rows, n->cols, 8, &a.x_ld) ||
      (n->residual && !take_ld(n->residual_ld, n->n_rows, n->cols, 8, &a.residual_ld)) ||
      (n->total && !take_ld(n->total_ld, n->n_rows, n->cols, 8, &a.total_ld)) ||
      (n->out && !take_ld(n->out_ld, n->n_rows, n->cols, 8, &a.out_ld)) ||
      (n->q && !take_ld(n->q_ld, n->n_rows, n->cols, 8, &a.q_ld)))
    return LLMCACHE_ERR_SHAPE;
  int dev = -1;
  Dev d;
  const cudaError_t e = ready(&dev, &d);
  if (e != cudaSuccess) return done(e);
  if (!pointer_on_device(n->x, dev)) return LLMCACHE_ERR_ARG;
  a.x = (const __nv_bfloat16*)n->x; a.residual = (const __nv_bfloat16*)n->residual;
  a.total = (__nv_bfloat16*)n->total; a.out = (__nv_bfloat16*)n->out;
  a.gain = n->gain; a.bias = n->bias;
  a.q = (uint8_t*)n->q; a.scale = n->scale;
  a.n_rows = n->n_rows; a.cols = n->cols; a.kind = n->kind; a.format = n->format;
  a.eps = n->eps > 0.f ? n->eps : 1e-5f;
  a.count_dev = n->count_dev; a.rows_per_count = n->rows_per_count ? n->rows_per_count : 1;
  return done(launch_norm(a, d.sm_count, (cudaStream_t)stream));
}

int llmcache_dense(const llmcache_dense_args* v, void* stream) {
  if (!v || v->struct_size != sizeof(llmcache_dense_args)) return LLMCACHE_ERR_ARG;
  if ((v->format != LLMCACHE_I8 && v->format != LLMCACHE_E4M3) || v->act > LLMCACHE_ACT_GELU_TANH) return LLMCACHE_ERR_ARG;
  if (v->n == 0 || v->k == 0 || v->k % 16 || v->k > 131056 || v->m > MOST_ROWS || v->n > MOST_ROWS) return LLMCACHE_ERR_SHAPE;
  if (((uint64_t)v->m + 127) / 128 * (((uint64_t)v->n + 63) / 64) > 0x7FFFFFFFull) return LLMCACHE_ERR_SHAPE;
  if (v->m == 0) return LLMCACHE_OK;
  const void* needed[] = {v->a, v->a_scale, v->w, v->w_scale, v->out};
  for (const void* p : needed)
    if (!p) return LLMCACHE_ERR_ARG;
  if (!aligned(v->a, 16) || !aligned(v->w, 16) || !aligned(v->out, 16) || !aligned(v->residual, 16) || !aligned(v->a_scale, 4) ||
      !aligned(v->w_scale, 16) || !aligned(v->bias, 16) || !aligned(v->count_dev, 4))
    return LLMCACHE_ERR_ARG;
  DenseArgs a{};
  if (!take_ld(v->a_ld, v->m, v->k, 16, &a.a_ld) || !take_ld(v->w_ld, v->n, v->k, 16, &a.w_ld) ||
      !take_ld(v->out_ld, v->m, v->n, 8, &a.out_ld) || (v->residual && !take_ld(v->residual_ld, v->m, v->n, 8, &a.residual_ld)))
    return LLMCACHE_ERR_SHAPE;
  int dev = -1;
  Dev d;
  const cudaError_t e = ready(&dev, &d);
  if (e != cudaSuccess) return done(e);
  if (!pointer_on_device(v->a, dev)) return LLMCACHE_ERR_ARG;
  a.a = (const uint8_t*)v->a; a.w = (const uint8_t*)v->w; a.a_scale = v->a_scale; a.w_scale = v->w_scale; a.bias = v->bias;
  a.residual = (const __nv_bfloat16*)v->residual; a.out = (__nv_bfloat16*)v->out;
  a.m = v->m; a.n = v->n; a.k = v->k; a.act = v->act; a.format = v->format;
  a.count_dev = v->count_dev; a.rows_per_count = v->rows_per_count ? v->rows_per_count : 1;
  a.status = d.status;
  if (d.form) {
    if (!form_serves(a, d.form)) return LLMCACHE_ERR_UNSUPPORTED;
    return done(d.form == LLMCACHE_DENSE_FEW ? launch_dense8_few(a, d.sm_count, (cudaStream_t)stream)
                                             : launch_dense8_tc(a, (int)d.form - LLMCACHE_DENSE_PAIRS, dev, d.sm_count, (cudaStream_t)stream));
  }
  return done(launch_dense8(a, d.sm_count, (cudaStream_t)stream));
}

int llmcache_dense_status(void) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) { cudaGetLastError(); return LLMCACHE_ERR_CUDA; }
  uint32_t *status = nullptr, s = 0;
  {
    std::lock_guard<std::mutex> lock(g_mu);
    if (!g_dev[dev].ready) return LLMCACHE_OK;               // never used on this device: nothing to report
    status = g_dev[dev].status;
  }
  if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&s, status, 4, cudaMemcpyDeviceToHost) != cudaSuccess) return done(cudaErrorUnknown);
  return s ? LLMCACHE_ERR_TIMEOUT : LLMCACHE_OK;
}

int llmcache_dense_debug_knobs(uint64_t wait_limit_ns, uint32_t flags) {
  const uint32_t form = flags >> 8 & 15u;
  if (form > LLMCACHE_DENSE_FEW) return LLMCACHE_ERR_ARG;
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) { cudaGetLastError(); return LLMCACHE_ERR_CUDA; }
  uint32_t* status = nullptr;
  {
    std::lock_guard<std::mutex> lock(g_mu);
    if (!g_dev[dev].ready) return LLMCACHE_ERR_STATE;
    g_dev[dev].form = form;
    status = g_dev[dev].status;
  }
  const uint32_t w[3] = {flags, (uint32_t)(wait_limit_ns & 0xFFFFFFFFull), (uint32_t)(wait_limit_ns >> 32)};
  if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(status + 1, w, sizeof(w), cudaMemcpyHostToDevice) != cudaSuccess) return done(cudaErrorUnknown);
  return LLMCACHE_OK;
}

}  // extern "C"
