// Internal launch interface of the dense operators of a target layer (include/fe_layer.h).
#pragma once

#include "fe_kernels.h"
#include "fe_layer.h"

namespace fe {

// What becomes of a matrix product z (and, GATED, of the second product u):
//   PLAIN       out = act(z + bias) + res, pre = z + bias
//   GATED       out = act(z) u, pre = z, pre2 = u
//   GATED_GRAD  of pre and pre2, as they were stored: out = z pre2 act'(pre), out2 = z act(pre), out3 = act(pre) pre2
enum FinishKind : int { FINISH_PLAIN = 0, FINISH_GATED = 1, FINISH_GATED_GRAD = 2 };
struct Finish {
    int kind, act;
    const void *bias, *res;
    int64_t res_row;
    void *out, *out2, *out3;
    int64_t out_row, out2_row, out3_row;
    float *pre, *pre2;
    int64_t pre_row, pre2_row;
    int vec;  // bias and all rows on 16-byte boundaries
};

// C [M, N] = sum over segments s of A_s [M, K] B_s [N, K]^T. An operand is stored as it is written
// here, or (t) with its K index as rows. FINISH_GATED: B_0 and B_1 belong to two products of A_0.
// twice: a second result A_1 B_0^T goes to e.out2.
struct GemmArgs {
    int64_t M;
    int N, K;
    int segs, twice;
    fe_mat a[2], b[2];
    int a_t, b_t;
    Finish e;
    int* status;
};

// d1 = dout act'(pre) (gated: dout pre2 act'(pre), and d2 = dout act(pre)), and d1's sums over the rows
struct ActGradArgs {
    int64_t M;
    int N, act, gated;
    fe_mat dout, pre, pre2;   // pre2, d2: gated only
    fe_mat d1, d2;            // d1 may be absent
    float* part;              // [parts][N] sums over the rows of each part, or NULL
    int parts, part_rows;
    int vec;
};

// The backward pass divides the rows among workers (CTAs, or warps of short rows): `parts` of them for
// each group of rows that share gates, or, where there are many groups, one for `step` whole groups.
struct NormArgs {
    int64_t R;
    int d, post;
    fe_mat x, z, gate;
    int64_t gate_rows;            // at most R
    const void *post_w, *pre_w;
    float scale, offset, eps;
    fe_mat y, n;                  // forward
    fe_mat dy, dn, dx, dz, dgate;  // backward
    int64_t groups, step;
    int parts;                    // 0: whole groups
    int gate_part;                // whether part_gate is needed for dgate (parts > 0: to be summed)
    float *part_post, *part_pre;  // [workers][d] sums over a worker's rows, or NULL
    float* part_gate;             // [workers][d], or NULL: a worker writes its groups' dgate itself
    int vec;
};

struct LogprobArgs {
    int64_t R;
    int V, J, K;
    fe_mat logits, dlogits;
    float temperature;
    const int* tokens;
    float *logprob, *entropy, *lse, *stats;
    int* top_id;
    float* top_logprob;
    const float *dlogprob, *dentropy, *dlse, *dtop;
    const int* top_in;
    const float *stats_in, *entropy_in;
    int* status;
};

cudaError_t launch_gemm_simt(const GemmArgs& a, int num_sms, cudaStream_t st);  // float32
cudaError_t launch_gemm_tc(const GemmArgs& a, int num_sms, cudaStream_t st);    // bfloat16
// whether launch_gemm_tc can read a matrix where it lies, and a copy that it can read
bool gemm_tc_reads(const fe_mat& m, int64_t rows, int64_t cols);
cudaError_t launch_pack_rows(const fe_mat& src, const fe_mat& dst, int64_t rows, int64_t cols, int num_sms, cudaStream_t st);
cudaError_t gemm_tc_prepare();
// the same for few rows of A: whether the kernel takes a product
bool gemm_few_takes(const GemmArgs& a);
cudaError_t launch_gemm_few(const GemmArgs& a, int num_sms, cudaStream_t st);
cudaError_t gemm_few_prepare();
// divides the rows into parts
void act_grad_plan(ActGradArgs& a, fe_dtype dtype, int num_sms);
cudaError_t launch_act_grad(const ActGradArgs& a, fe_dtype dtype, cudaStream_t st);
// row g of out [groups, n] = sum over i < parts of part[g][i][n], in order, rounded to the type
struct SumJob {
    const float* part;
    int64_t parts, groups;
    void* out;
    int64_t out_row;
};
struct SumJobs {
    SumJob job[3];
    int jobs;
    int64_t n;
    void add(const float* part, int64_t parts, int64_t groups, void* out, int64_t out_row) {
        job[jobs++] = SumJob{part, parts, groups, out, out_row};
    }
};
cudaError_t launch_sum_parts(const SumJobs& a, fe_dtype dtype, cudaStream_t st);
cudaError_t norm_prepare(fe_dtype dtype);
cudaError_t launch_block_norm(const NormArgs& a, fe_dtype dtype, int num_sms, cudaStream_t st);
// fills in how the rows are divided (by what norm_backward_prepare has asked of the device, or a guess where there is
// none), and returns the number of workers: rows of part_post and part_pre
int64_t norm_backward_plan(NormArgs& a, fe_dtype dtype, int num_sms);
cudaError_t norm_backward_prepare(fe_dtype dtype);
cudaError_t launch_block_norm_backward(const NormArgs& a, fe_dtype dtype, cudaStream_t st);
cudaError_t launch_token_logprobs(const LogprobArgs& a, fe_dtype dtype, int num_sms, cudaStream_t st);
cudaError_t launch_token_logprobs_backward(const LogprobArgs& a, fe_dtype dtype, int num_sms, cudaStream_t st);
cudaError_t logprobs_prepare(fe_dtype dtype);

}  // namespace fe
