// Rotation of queries and keys by position: shared declarations.
#pragma once
#include "attn.cuh"

namespace llmc {

// llmcache_rotation, checked; dims 0: nothing turns
struct RotateArgs { const double* inv_freq; uint32_t dims, interleaved; };

// llmcache_rotation -> RotateArgs (nullptr: dims 0) or an error status
int check_rotation(const llmcache_rotation* r, RotateArgs* o);
// the checks of llmcache_kv_append alone
int kv_check_append(const llmcache_kv* kv, const llmcache_kv_new* c);
// llmcache_kv_append; rotate: a rotation that was checked before, in place of c's
int kv_append(llmcache_kv* kv, const llmcache_kv_new* c, const RotateArgs* rotate, cudaStream_t st);

// a.out: where a.q goes.  With pages: a.k and a.v are the new rows of a paged call; without: a.q and a.k hold n_rows rows of sequences of a.n
// tokens (a.n_seqs_dev of them where given), and k is turned in its place.
cudaError_t launch_kv_rotate(const AttnArgs& a, const RotateArgs& r, int sm_count, cudaStream_t st);

}  // namespace llmc
