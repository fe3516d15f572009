// The target-side handle (include/fe_target.h) and what every entry point on it does first.
#pragma once

#include <stdio.h>

#include <atomic>

#include "fe_target_kernels.h"

struct fe_target {
    fe_target_config cfg;
    int device = 0, num_sms = 0;
    float2* rope = nullptr;
    float *part_o = nullptr, *part_ml = nullptr;
    int* status = nullptr;
    fe::SplitDesc* split = nullptr;
    mutable std::atomic<unsigned> ready{0};  // kernels of the dense operators that are set up (fe::Kernels)
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

// What the dense operators need of the device before their kernels run (shared memory above 48 KB, large clusters, how
// many CTAs fit) is asked for when a handle first uses them: it loads their modules, 17 ms in a process (16 of them the
// norms'), which a handle that only rotates and attends need not pay. Twice, from two threads, does no harm.
enum Kernels : unsigned { GEMM_TC = 1, GEMM_FEW = 2, NORM = 4, NORM_BACKWARD = 8, LOGPROBS_F32 = 16, LOGPROBS_BF16 = 32 };
template <typename F>
fe_status set_up(const fe_target* t, Kernels which, const F& prepare) {
    if (t->ready.load(std::memory_order_acquire) & which) return FE_OK;
    int dev = -1;
    FE_TRY(cudaGetDevice(&dev));
    FE_TRY(prepare());
    if (dev == t->device) t->ready.fetch_or(which, std::memory_order_release);
    return FE_OK;
}
#undef FE_SOURCE

}  // namespace fe
