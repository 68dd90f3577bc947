// Host-side construction of TMA tensor maps.
#include "llmcache_internal.cuh"
#include "ptx.cuh"
#include "attn.cuh"

namespace llmc {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiledFn g_encode = nullptr;
typedef CUresult (*PointerAttributeFn)(void*, CUpointer_attribute, CUdeviceptr);
static PointerAttributeFn g_pointer = nullptr;

cudaError_t tensor_map_setup() {
  if (g_encode) return cudaSuccess;
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult q;
  cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q);
  if (e != cudaSuccess) return e;
  if (!fn || q != cudaDriverEntryPointSuccess) return cudaErrorNotSupported;
  void* pointer = nullptr;
  e = cudaGetDriverEntryPoint("cuPointerGetAttribute", &pointer, cudaEnableDefault, &q);
  if (e != cudaSuccess) return e;
  if (!pointer || q != cudaDriverEntryPointSuccess) return cudaErrorNotSupported;
  g_pointer = (PointerAttributeFn)pointer;
  g_encode = (EncodeTiledFn)fn;
  return cudaSuccess;
}

bool pointer_on_device(const void* p, int device) {
  int at = -1;
  return g_pointer && g_pointer(&at, CU_POINTER_ATTRIBUTE_DEVICE_ORDINAL, (CUdeviceptr)p) == CUDA_SUCCESS && at == device;
}

bool make_tensor_map_bf16(CUtensorMap* map, const void* ptr, uint64_t rows, uint64_t k, uint32_t box_rows) {
  return make_tensor_map_bf16_pitch(map, ptr, rows, k, k, box_rows);
}

bool make_tensor_map_bf16_pitch(CUtensorMap* map, const void* ptr, uint64_t rows, uint64_t k, uint64_t pitch,
                                uint32_t box_rows) {
  if (!g_encode) return false;
  const cuuint64_t dims[2] = {k, rows};
  const cuuint64_t strides[1] = {pitch * 2};
  const cuuint32_t box[2] = {64u, box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return g_encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(ptr), dims, strides, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool make_tensor_map_bf16_box32(CUtensorMap* map, const void* ptr, uint64_t rows, uint64_t cols) {
  if (!g_encode) return false;
  const cuuint64_t dims[2] = {cols, rows};
  const cuuint64_t strides[1] = {cols * 2};
  const cuuint32_t box[2] = {32u, 32u};
  const cuuint32_t estr[2] = {1, 1};
  return g_encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(ptr), dims, strides, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool make_tensor_map_rows(CUtensorMap* map, const RowsArgs& r, uint64_t heads, uint64_t toks, uint64_t seqs, uint32_t box_heads,
                          uint32_t box_toks) {
  if (!g_encode) return false;
  // (the stride of a dimension of size one is never used: any valid one will do)
  const cuuint64_t dims[4] = {64, heads, toks, seqs};
  const cuuint64_t strides[3] = {heads > 1 ? (cuuint64_t)r.head * 2 : 128, toks > 1 ? (cuuint64_t)r.tok * 2 : 128,
                                 seqs > 1 ? (cuuint64_t)r.seq * 2 : 128};
  const cuuint32_t box[4] = {64u, box_heads, box_toks, 1u};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return g_encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, r.ptr, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace llmc
