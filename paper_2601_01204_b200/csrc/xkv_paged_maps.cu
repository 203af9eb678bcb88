// Tensor maps of the pools and of token tensors.
#include "xkv_paged_internal.cuh"

namespace xkv {

namespace {

typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                           const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

Encode find_encode() {
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess) return nullptr;
  return found == cudaDriverEntryPointSuccess ? reinterpret_cast<Encode>(fn) : nullptr;
}

// 16-bit elements, 64 channels (128 bytes) a row, swizzled over 128 bytes.
cudaError_t encode(CUtensorMap* map, int dtype, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  static const Encode fn = find_encode();
  if (!fn) return cudaErrorNotSupported;
  const cuuint32_t one[4] = {1, 1, 1, 1};
  const CUresult r = fn(map, dtype == XKV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank, const_cast<void*>(base),
                        dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace

cudaError_t make_pool_maps(const PagedView& c, int head_dim, int dtype, int rows, PoolMaps* maps) {
  const cuuint64_t dims[4] = {(cuuint64_t)head_dim, (cuuint64_t)1 << c.page_shift, (cuuint64_t)c.n_kv_heads, (cuuint64_t)c.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)c.slot_stride * 2, (cuuint64_t)c.head_stride * 2, (cuuint64_t)c.page_stride * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)rows, 1, 1};
  const cudaError_t e = encode(&maps->k, dtype, 4, c.k, dims, strides, box);
  return e != cudaSuccess ? e : encode(&maps->v, dtype, 4, c.v, dims, strides, box);
}

cudaError_t make_token_map(const void* base, int64_t ts, int64_t hs, int n, int n_heads, int head_dim, int dtype, int heads, int toks,
                           CUtensorMap* map) {
  const cuuint64_t dims[3] = {(cuuint64_t)head_dim, (cuuint64_t)n_heads, (cuuint64_t)n};
  const cuuint64_t strides[2] = {(cuuint64_t)hs * 2, (cuuint64_t)ts * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)heads, (cuuint32_t)toks};
  return encode(map, dtype, 3, base, dims, strides, box);
}

}  // namespace xkv
