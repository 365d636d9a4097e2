// Host-side construction of TMA tensor maps (the driver's encoder, reached through the runtime).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

namespace crf {

using TensorMapEncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                       const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                       CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                       CUtensorMapFloatOOBfill);

inline TensorMapEncodeFn tensor_map_encode() {
  static TensorMapEncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      return reinterpret_cast<TensorMapEncodeFn>(p);
    return static_cast<TensorMapEncodeFn>(nullptr);
  }();
  return fn;
}

// bf16 [rows, cols] row-major (cols elements apart), box of box_rows x 64 columns in the
// 128-byte-swizzled layout; elements outside the matrix read as zero.
inline bool tensor_map_rows(CUtensorMap* m, const void* base, long rows, int cols, int box_rows) {
  TensorMapEncodeFn fn = tensor_map_encode();
  if (!fn) return false;
  cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  cuuint64_t strides[1] = {static_cast<cuuint64_t>(cols) * 2};
  cuuint32_t box[2] = {64, static_cast<cuuint32_t>(box_rows)};
  cuuint32_t estr[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// K or V pool of one layer, [rows = pages * Hkv * 16, D] row-major, as the 4-D view
// {64 columns, 8 rows, D/64 halves, rows/8 groups} with strides {2D, 128, 16D} bytes; the box
// {64, 8, D/64, 2} is one page of one kv head, written to shared memory group-major, halves
// inside a group, each half an 8 x 128-byte swizzled atom.
inline bool tensor_map_pool(CUtensorMap* m, const void* base, long rows, int D) {
  TensorMapEncodeFn fn = tensor_map_encode();
  if (!fn) return false;
  cuuint64_t dims[4] = {64, 8, static_cast<cuuint64_t>(D / 64), static_cast<cuuint64_t>(rows / 8)};
  cuuint64_t strides[3] = {static_cast<cuuint64_t>(D) * 2, 128, static_cast<cuuint64_t>(D) * 16};
  cuuint32_t box[4] = {64, 8, static_cast<cuuint32_t>(D / 64), 2};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box,
            estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace crf
