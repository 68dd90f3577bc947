// Attention operators: what their host code shares with the layer's.
#pragma once
#include "attn.cuh"

struct llmcache_kv {
  llmcache_kv_desc desc{};
  int sm_count = 0;
  char* ws = nullptr;
  bool owns_ws = false;
  uint32_t* status = nullptr;    // a bounded wait expired; diagnostic knobs behind it
  float* part = nullptr;         // shares of the keys of one call
  uint32_t* arrived = nullptr;   // [max_seqs, kv_heads], zero between calls
  float* scores = nullptr;       // of few rows whose weights are recorded: score_floats of them
  size_t score_floats = 0;
  float2* stat = nullptr;        // [max_rows, heads] of a call that records weights
  int32_t* kept = nullptr;       // eviction: slots kept [max_seqs, kv_heads, <= max_len] ...
  uint32_t* count = nullptr;     // ... and how many per sequence
};

namespace llmc {

// llmcache_score_mods -> ScoreArgs (nullptr: plain, not causal) or an error status
int check_score_mods(const llmcache_score_mods* m, ScoreArgs* o);
// whether a layer of `heads` heads on `device` can keep its keys and values in kv
int kv_fits_layer(const llmcache_kv* kv, int device, uint32_t heads);

// the checks of llmcache_kv_attention alone
int kv_check_chunk(const llmcache_kv* kv, const llmcache_kv_chunk* c);
// llmcache_kv_attention; zero_rest: zeros in the rows of out that `longest` leaves out
int kv_attend(llmcache_kv* kv, const llmcache_kv_chunk* c, bool zero_rest, cudaStream_t st);

// launch_attn behind the check of its grid
inline int launch_attn_checked(const AttnArgs& a, const AttnScratch& s, int sm_count, cudaStream_t st) {
  const uint64_t tiles = ((uint64_t)a.n * a.group + 127) / 128 * a.kv_heads * a.n_seqs;
  if (tiles > 0x7FFFFFFFull) return LLMCACHE_ERR_SHAPE;
  if (launch_attn(a, s, sm_count, st) == cudaSuccess) return LLMCACHE_OK;
  cudaGetLastError();
  return LLMCACHE_ERR_CUDA;
}

}  // namespace llmc
