// Runs the join of split attention items (fe_tree_attn_join.cuh) alone, on notes and partial results
// of the caller's: one sequence, `T` nodes, two heads of 64 float32 columns, `ncta` CTAs of 64 rows.
#include "fe_tree_attn_join.cuh"

using namespace fe;

extern "C" __attribute__((visibility("default"))) int join_notes(int T, int ncta, float* out, float* lse, const int* prefix,
                                                                 void* notes, float* part_o, float* part_ml, int* status) {
    TreeAttnArgs a{};
    a.B = 1;
    a.T = T;
    a.H = a.Hkv = 2;
    a.G = 1;
    a.out = fe_rows{out, (int64_t)T * 128, 128, 64};
    a.lse = lse;
    a.prefix = prefix;
    a.cache.max_seq = 1 << 20;
    a.cache.Hkv = 2;
    a.split = (SplitDesc*)notes;
    a.part_rows = 64;
    a.part_o = part_o;
    a.part_ml = part_ml;
    a.status = status;
    a.out_vec = 1;
    const int rows = (T < 64 ? T : 64) + 31;
    const cudaError_t e = launch_k(tree_attn_join_kernel<float, 64, 64>, dim3(ncta, (rows / 32 * 4 + kJoinWarps - 1) / kJoinWarps),
                                   dim3(kJoinThreads), 0, nullptr, false, a);
    return (int)(e != cudaSuccess ? e : cudaDeviceSynchronize());
}

extern "C" __attribute__((visibility("default"))) int note_bytes() { return (int)sizeof(SplitDesc); }
