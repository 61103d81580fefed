// Tensor maps (the descriptors of tiled TMA copies) of the floating-point products, made on the host.
#pragma once

#include <cuda.h>

#include "common.cuh"

namespace qb {

typedef CUresult (*TensormapEncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline qb_status tensormap_encoder(TensormapEncodeFn* out) {
  static TensormapEncodeFn cached = nullptr;
  if (!cached) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult qres;
    QB_CUDA_TRY(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres));
    if (qres != cudaDriverEntryPointSuccess || !fn) {
      set_last_error("cuTensorMapEncodeTiled not available from the driver");
      return QB_ERR_CUDA;
    }
    cached = reinterpret_cast<TensormapEncodeFn>(fn);
  }
  *out = cached;
  return QB_OK;
}

// A row-major matrix [rows][cols] whose rows begin `row_bytes` apart; boxes of box_rows x box_cols elements.  base and row_bytes
// are multiples of 16; what a box has outside the matrix reads as zero and is not written.
inline qb_status make_matrix_map(CUtensorMap* tm, CUtensorMapDataType type, const void* base, int64_t rows, int64_t cols,
                                 int64_t row_bytes, int box_rows, int box_cols, CUtensorMapSwizzle swizzle,
                                 CUtensorMapL2promotion promotion = CU_TENSOR_MAP_L2_PROMOTION_L2_128B) {
  TensormapEncodeFn encode = nullptr;
  qb_status st = tensormap_encoder(&encode);
  if (st != QB_OK) return st;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)row_bytes};
  const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows};
  const cuuint32_t elem[2] = {1, 1};
  const CUresult r = encode(tm, type, 2, const_cast<void*>(base), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                            promotion, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    set_last_error("cuTensorMapEncodeTiled failed with CUresult %d (%lld x %lld)", (int)r, (long long)rows, (long long)cols);
    return QB_ERR_CUDA;
  }
  return QB_OK;
}

// The same matrix as column groups of 128 bytes: coordinates (byte in the group, row, group), boxes of box_rows rows x box_groups
// groups, 128-byte swizzle.  row_bytes is a multiple of 128 here (a group's part behind a row's end would be the next row's).
inline qb_status make_group_map(CUtensorMap* tm, CUtensorMapDataType type, int esize, const void* base, int64_t rows, int64_t row_bytes,
                                int box_rows, int box_groups) {
  TensormapEncodeFn encode = nullptr;
  qb_status st = tensormap_encoder(&encode);
  if (st != QB_OK) return st;
  const cuuint64_t dims[3] = {(cuuint64_t)(128 / esize), (cuuint64_t)rows, (cuuint64_t)(row_bytes / 128)};
  const cuuint64_t strides[2] = {(cuuint64_t)row_bytes, 128};
  const cuuint32_t box[3] = {(cuuint32_t)(128 / esize), (cuuint32_t)box_rows, (cuuint32_t)box_groups};
  const cuuint32_t elem[3] = {1, 1, 1};
  const CUresult r = encode(tm, type, 3, const_cast<void*>(base), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    set_last_error("cuTensorMapEncodeTiled failed with CUresult %d (%lld rows of %lld bytes)", (int)r, (long long)rows, (long long)row_bytes);
    return QB_ERR_CUDA;
  }
  return QB_OK;
}

// `parts` matrices one after the other, row-major without gaps: coordinates (column, row, part), boxes of one part.
inline qb_status make_parts_map(CUtensorMap* tm, CUtensorMapDataType type, const void* base, int64_t parts, int64_t rows, int64_t cols,
                                int64_t row_bytes, int box_rows, int box_cols, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
  TensormapEncodeFn encode = nullptr;
  qb_status st = tensormap_encoder(&encode);
  if (st != QB_OK) return st;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)parts};
  const cuuint64_t strides[2] = {(cuuint64_t)row_bytes, (cuuint64_t)(rows * row_bytes)};
  const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1};
  const cuuint32_t elem[3] = {1, 1, 1};
  const CUresult r = encode(tm, type, 3, const_cast<void*>(base), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            swizzle, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    set_last_error("cuTensorMapEncodeTiled failed with CUresult %d (%lld x %lld x %lld)", (int)r, (long long)parts, (long long)rows, (long long)cols);
    return QB_ERR_CUDA;
  }
  return QB_OK;
}

}  // namespace qb
