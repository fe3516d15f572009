// Whether the attention's schedules take a shape (fe_attn_plan.cuh), for the host.
#include "fe_attn_plan.cuh"

extern "C" __attribute__((visibility("default"))) int plan_fits(int dtype, int cache_dtype, int B, int Hkv, int T, int G, int max_seq) {
    return fe::attn_plan_fits((fe_dtype)dtype, (fe_dtype)cache_dtype, B, Hkv, T, G, max_seq);
}
