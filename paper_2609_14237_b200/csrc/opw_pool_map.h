// Tensor maps of the layers' pools, for the kernels that copy key and value tiles by TMA.
#pragma once
#include <cstdint>
#include <vector>

#include <cuda.h>
#include <cuda_runtime.h>

#include "opw_stage.h"

typedef CUresult (*opw_tensor_map_fn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                      const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                      CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// One layer's pool as [page and head][K, V][slot][64 dimensions at a time][64]; a box is 16 slots of 64 dimensions.  No
// swizzle: the pool's own permutation is the one the tensor core expects.
inline bool opw_encode_pool(opw_tensor_map_fn fn, CUtensorMap* map, void* pool, const opw_stage_view& v, int64_t num_pages) {
  const cuuint64_t row = (cuuint64_t)v.D * 2;
  const cuuint64_t dims[5] = {64, (cuuint64_t)v.D / 64, 16, 2, (cuuint64_t)num_pages * v.Hkv};
  const cuuint64_t strides[4] = {128, row, 16 * row, 32 * row};
  const cuuint32_t box[5] = {64, 1, 16, 1, 1}, elem[5] = {1, 1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, pool, dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// One map per layer.
inline opw_status_t opw_map_pools(const opw_stage_view& v, std::vector<CUtensorMap>* maps) {
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found);
  if (e != cudaSuccess || found != cudaDriverEntryPointSuccess || !fn) { (void)cudaGetLastError(); return OPW_ERR_CUDA; }
  try {
    maps->resize(v.num_layers);
  } catch (...) {
    return OPW_ERR_INVALID_ARG;
  }
  for (size_t i = 0; i < maps->size(); ++i)
    if (!opw_encode_pool(reinterpret_cast<opw_tensor_map_fn>(fn), &(*maps)[i], v.pool[i], v, v.num_pages[i])) return OPW_ERR_CUDA;
  return OPW_OK;
}
