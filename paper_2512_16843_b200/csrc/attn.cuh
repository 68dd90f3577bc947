// Attention operators (score modifiers, paged key/value cache, eviction): shared declarations.
#pragma once
#include "llmcache_internal.cuh"

namespace llmc {

constexpr float LOG2E_F = 1.4426950408889634f;
constexpr float LN2_F = 0.6931471805599453f;

// llmcache_score_mods, checked; positions are those of the header
struct ScoreArgs {
  float scale, cap;
  uint32_t causal;
  int32_t reach;
  const float* slopes;
  const float* table;
  const int32_t* doc;
  const int32_t* prefix;
  uint32_t mask_seqs;            // entries of doc and prefix; 0: unknown
};

struct RowsArgs {
  __nv_bfloat16* ptr;
  long long seq, tok, head;      // strides in elements
};

// One call of the attention over whole sequences (pages == nullptr) or over a paged cache.
struct AttnArgs {
  RowsArgs q, out, k, v;         // paged: k, v are the new rows (ptr may be null), seq strides unused
  float* lse;                    // or null
  float2* stat;                  // calls that record weights: (maximum, sum) of a row's exponentials, base 2 [n_rows, heads]; or null
  uint32_t heads, kv_heads, group, n_seqs;
  const uint32_t* n_seqs_dev;
  ScoreArgs m;
  uint32_t* status;
  uint32_t n;                    // whole sequences: tokens of one; paged: most rows of one sequence
  // paged
  const int32_t *cu, *lens, *pages, *first;
  int32_t* positions;
  float* weights;
  float decay;
  uint32_t n_rows, pages_ld, num_pages, page_shift, max_len;
  unsigned long long side_ld, page_stride;
  __nv_bfloat16 *k_pages, *v_pages;
  // few rows whose weights are asked for: modified scores (base 2, -inf: not seen) [n_seqs, kv_heads, row][score_ld], or null
  float* scores;
  uint32_t score_ld, score_rows;
  // rows of a sequence beyond the n that are computed get zeros in out (they are left as they were otherwise)
  uint32_t zero_rest;
};

// A sequence of a paged call: its rows row0 .. row0 + all - 1 take the slots slot0 .. of len slots; the first cnt of them
// are computed, the others stored only.  Whatever the arrays hold, rows stay inside [0, n_rows) and slots inside the page
// table.
struct SeqGeo { uint32_t row0, cnt, len; int32_t slot0; uint32_t all; };
__device__ __forceinline__ SeqGeo seq_geo(const AttnArgs& a, uint32_t s) {
  SeqGeo g;
  const int32_t c0 = a.cu[s], c1 = a.cu[s + 1], len = a.lens[s];
  const uint32_t cap = min((unsigned long long)a.max_len, (unsigned long long)a.pages_ld << a.page_shift);
  g.len = len > 0 ? min((uint32_t)len, cap) : 0u;
  const bool sane = c0 >= 0 && c1 >= c0 && (uint32_t)c1 <= a.n_rows;
  g.row0 = sane ? (uint32_t)c0 : 0u;
  g.all = sane ? (uint32_t)(c1 - c0) : 0u;
  g.slot0 = (int32_t)g.len - (int32_t)g.all;
  g.cnt = min(g.all, a.n);
  return g;
}
// page of a slot, or -1 where the table has none
__device__ __forceinline__ int32_t page_of(const AttnArgs& a, uint32_t s, uint32_t slot) {
  const int32_t p = a.pages[(size_t)s * a.pages_ld + (slot >> a.page_shift)];
  return (uint32_t)p < a.num_pages ? p : -1;
}
__device__ __forceinline__ size_t page_row(const AttnArgs& a, int32_t page, uint32_t hk, uint32_t slot) {
  return (size_t)page * a.page_stride + (((size_t)hk << a.page_shift) + (slot & ((1u << a.page_shift) - 1u))) * 64;
}

// sequence whose rows include `row`: the last one whose first row is not behind it
__device__ __forceinline__ uint32_t seq_of_row(const AttnArgs& a, uint32_t row) {
  uint32_t lo = 0, hi = a.n_seqs;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (a.cu[mid] <= (int32_t)row) lo = mid; else hi = mid;
  }
  return lo;
}

constexpr size_t PART_FLOATS = 66;                 // one (row, head, share of the keys): 64 sums, the maximum, the sum of weights
constexpr uint32_t ATTN_MAX_GROUP = 128;           // query heads per key/value head: rows of one query tile
cudaError_t setup_attn_tc();
cudaError_t launch_attn_tc(const AttnArgs& a, float* part, size_t part_units, int sm_count, cudaStream_t st);
constexpr uint32_t FEW_ROWS = 16;                  // rows of a sequence and key/value head that k_attn_few takes
// Whether a paged call goes to k_attn_few: at most 16 rows per sequence and key/value head.  It stores the new rows itself.
bool attn_is_few(const AttnArgs& a);
cudaError_t setup_attn_few();
size_t attn_few_part_floats(int sm_count);
cudaError_t launch_attn_few(const AttnArgs& a, float* part, uint32_t* arrived, int sm_count, cudaStream_t st);
cudaError_t setup_attn_kernels();
// Scratch of a paged call: part for part_units x PART_FLOATS floats, arrived for [n_seqs, kv_heads] words that are zero
// between calls.  Null for whole sequences.
struct AttnScratch {
  float* part = nullptr;
  size_t part_units = 0;
  uint32_t* arrived = nullptr;
};
cudaError_t launch_attn(const AttnArgs& a, const AttnScratch& s, int sm_count, cudaStream_t st);
// received weights of a paged call whose stat is complete
cudaError_t launch_attn_weights(const AttnArgs& a, int sm_count, cudaStream_t st);
cudaError_t launch_kv_append(const AttnArgs& a, int sm_count, cudaStream_t st);

struct EvictArgs {
  uint32_t n_seqs, kv_heads, budget, recent, sinks, pages_ld, new_pages_ld, num_pages, page_shift, max_len;
  unsigned long long side_ld, new_side_ld, page_stride;
  const int32_t *lens, *pages, *new_pages;
  int32_t* new_lens;
  const float* weights;
  const int32_t* positions;
  float* new_weights;
  int32_t* new_positions;
  int32_t* kept_out;             // optional
  int32_t* kept;                 // scratch [n_seqs, kv_heads, budget]
  uint32_t* count;               // scratch [n_seqs]
  __nv_bfloat16 *k_pages, *v_pages;
};
cudaError_t setup_evict_kernels();
cudaError_t launch_evict_tokens(const EvictArgs& a, int sm_count, cudaStream_t st);

}  // namespace llmc
