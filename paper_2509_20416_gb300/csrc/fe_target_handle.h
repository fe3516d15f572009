// The target-side handle (include/fe_target.h) and what every entry point on it does first.
#pragma once

#include <stdio.h>

#include "fe_target_kernels.h"

struct fe_target {
    fe_target_config cfg;
    int device = 0, num_sms = 0;
    float2* rope = nullptr;
    float *part_o = nullptr, *part_ml = nullptr;
    int* status = nullptr;
    fe::SplitDesc* split = nullptr;
};

namespace fe {

inline fe_status fail(cudaError_t e, const char* what, const char* file) {
    char buf[200];
    snprintf(buf, sizeof(buf), "%s (%s): %s", what, file, cudaGetErrorString(e));
    set_error_detail(buf);
    return e == cudaErrorMemoryAllocation ? FE_ERR_OOM : FE_ERR_CUDA;
}

// the call, or its CUDA error as the entry point's status (FE_SOURCE: the file, for the detail string)
#define FE_TRY(call)                                                 \
    do {                                                             \
        cudaError_t _e = (call);                                     \
        if (_e != cudaSuccess) return ::fe::fail(_e, #call, FE_SOURCE); \
    } while (0)

#define FE_SOURCE "fe_target_handle.h"
inline fe_status check_device(const fe_target* t) {
    int dev = -1;
    FE_TRY(cudaGetDevice(&dev));
    if (dev == t->device) return FE_OK;
    char buf[128];
    snprintf(buf, sizeof(buf), "the current CUDA device (%d) is not the handle's device (%d)", dev, t->device);
    set_error_detail(buf);
    return FE_ERR_INVALID_ARG;
}
#undef FE_SOURCE

}  // namespace fe
