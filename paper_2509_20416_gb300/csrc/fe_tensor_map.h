// Tensor maps for TMA copies, encoded on the host.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

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

}  // namespace fe
