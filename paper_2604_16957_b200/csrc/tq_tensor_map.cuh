// Tensor maps of packed heads (internal): host side.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include "tq.h"

namespace tq {

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeFn encode_fn() {
  static const EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      return static_cast<EncodeFn>(nullptr);
    }
    return reinterpret_cast<EncodeFn>(p);
  }();
  return fn;
}

// [rows][heads][d] values, rows `stride` elements apart and heads `head`, boxes of 128 bytes x `heads_box` x `rows_box`
inline bool make_map(CUtensorMap* map, const void* p, int dtype, int d, int heads, long long rows, long long stride, long long head, int heads_box,
              int rows_box) {
  const int size = dtype == TQ_FP32 ? 4 : 2;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(head) * size, static_cast<cuuint64_t>(stride) * size};
  const cuuint32_t box[3] = {128u / size, static_cast<cuuint32_t>(heads_box), static_cast<cuuint32_t>(rows_box)};
  const cuuint32_t ones[3] = {1, 1, 1};
  const CUtensorMapDataType type = dtype == TQ_FP32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == TQ_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                      : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return encode_fn()(map, type, 3, const_cast<void*>(p), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace tq
