// Tensor maps for TMA copies, encoded on the host.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include "fe_layer.h"

namespace fe {

// cuTensorMapEncodeTiled, looked up once (the library does not link the driver)
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiled encode_tiled() {
    static const EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &r) != cudaSuccess) return (EncodeTiled) nullptr;
        return r == cudaDriverEntryPointSuccess ? (EncodeTiled)p : nullptr;
    }();
    return fn;
}

// A matrix [rows, cols] of bfloat16 in boxes of 64 columns, 128-byte swizzled; beyond its edges zeros
inline bool tensor_map_bf16(CUtensorMap* map, const fe_mat& m, int64_t rows, int64_t cols, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(rows > 1 ? m.row : (cols + 7) / 8 * 8) * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, step[2] = {1, 1};
    const EncodeTiled encode = encode_tiled();
    return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, m.p, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace fe
