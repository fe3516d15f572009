// How matrix products are divided (fe_gemm_plan.h), for the host.
#include "fe_gemm_plan.h"

#define EXPORT extern "C" __attribute__((visibility("default")))

// out: width, tiles, slices in flight
EXPORT void gemm_tc_plan(int64_t M, int N, int gated, int twice, int grad, int b_t, int num_sms, int64_t* out) {
    const fe::TcWidth w = fe::tc_width(M, N, gated, twice, grad, b_t, num_sms);
    out[0] = w.bn;
    out[1] = fe::tc_tiles(M, N, gated, twice, w.bn);
    out[2] = w.stages;
    out[3] = (int64_t)w.stages * (fe::kSliceA + w.b_bytes);
}

// out: CTAs of a block, slices in flight, bytes of shared memory
EXPORT void gemm_few_plan(int64_t M, int N, int K, int gated, int num_sms, int64_t* out) {
    int smem = 0;
    const fe::FewArgs f = fe::few_plan(M, N, K, gated, num_sms, &smem);
    out[0] = f.ranks;
    out[1] = f.stages;
    out[2] = smem;
}

EXPORT int gemm_simt_large(int64_t M, int N, int gated, int twice, int num_sms) { return fe::simt_large(M, N, gated, twice, num_sms); }
