// Tensor maps for tiled copies of rows of heads: dims {inner, heads, rows}, a box of 64 x box_heads x box_rows values with the 128-byte swizzle.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

namespace pask {

inline bool encode_heads(CUtensorMap *map, const void *base, int inner, int heads, int rows, size_t head_stride, size_t row_stride, int box_heads,
                         int box_rows) {
    using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                     const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                     CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const EncodeTiled fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found);
        return reinterpret_cast<EncodeTiled>(e == cudaSuccess && found == cudaDriverEntryPointSuccess ? f : nullptr);
    }();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)inner, (cuuint64_t)heads, (cuuint64_t)rows}, strides[2] = {head_stride, row_stride};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows}, one[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace pask
