/*
 * fe_layer.h -- C ABI of the dense part of a target layer and of the target's answer, next to the
 * operators of fe_target.h on the same handle (sm_103a):
 *
 *   fe_project         act(x w^T + bias) + residual
 *   fe_gated_ffn       act(x w_gate^T) * (x w_up^T), the gated half of a feed-forward block
 *   fe_block_norm      y = x + scale gate norm(z), n = norm(y): the norms behind a block and before
 *                      the next, with the block's gate and residual
 *   fe_token_logprobs  log probabilities of given tokens, the entropy, the most probable tokens
 *
 * each with its gradients (the calls named _backward). A layer is fe_block_norm, fe_project
 * (query, key and value rows), fe_cache_write and fe_tree_attention, fe_project, fe_block_norm,
 * fe_gated_ffn and fe_project with the residual; the head is fe_project, and fe_token_logprobs
 * reads its logits (top_id's first column is fe_verify_greedy's target_next).
 *
 * The conventions of fe_target.h hold. All tensors have the handle's type (dtype: FE_F32 or
 * FE_BF16) unless stated, every product, sum and statistic is accumulated in float32, and a
 * result is rounded once. Matrices need no alignment beyond their type's own; rows on 16-byte
 * boundaries (the address and the row stride) are faster. Outputs must not overlap inputs or one
 * another except where stated. Calls that take `work` need device memory of at least the
 * bytes that the call's _work function returns for the same arguments (it looks at `work` and
 * `work_bytes` not at all; 0: none needed; a negative fe_status for arguments that the call
 * refuses), on a 256-byte boundary and theirs alone until they have run: calls with a workspace
 * each may run at once. Calls without rows (M or R of 0) write the weights' gradients, as zeros,
 * and nothing else.
 * The result does not depend on timing: the same call gives the same bits.
 * A handle sets up the kernels of an operator when it is first called (on the host; a process's first norm takes 16 ms,
 * the others less than one; a stream may be capturing).
 */
#ifndef FE_LAYER_H
#define FE_LAYER_H

#include "fe_target.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A matrix with contiguous columns: row i starts at p + i * row elements. row >= columns for
 * outputs of more than one row; inputs may repeat a row (0). p == NULL: not given. */
typedef struct {
    void *p;
    int64_t row;
} fe_mat;

/* act(z): z; max(z, 0) (gradient 0 at 0); z / (1 + e^-z); z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2 */
typedef enum { FE_ACT_NONE = 0, FE_ACT_RELU = 1, FE_ACT_SILU = 2, FE_ACT_GELU = 3 } fe_act;

/* out [M, N] = act(x [M, K] w [N, K]^T + bias [N]) + residual [M, N].
 *  bias, residual  may be absent; out may be the residual itself (the same p and row)
 *  pre             float32 [M, N] or absent: x w^T + bias, which the gradient of an activation needs
 * M >= 0 up to 2^30; N, K in 1..2^24. */
typedef struct {
    int64_t M;
    int32_t N, K;
    fe_mat x, w;
    const void *bias;
    fe_mat residual, out, pre;
    fe_act act;
    void *work;
    int64_t work_bytes;
} fe_project_args;
FE_API int64_t fe_project_work(const fe_target *t, const fe_project_args *a);
FE_API fe_status fe_project(fe_target *t, const fe_project_args *a, void *stream);

/* Gradients of fe_project for dout [M, N] (the residual's is dout itself), pre as fe_project stored it:
 * with dz = dout act'(pre), rounded to the handle's type where act is not NONE,
 *   dx [M, K] = dz w,  dw [N, K] = dz^T x,  dbias [N] = sum over rows of dz;
 * each may be absent. w is read for dx, x for dw, pre for act != NONE. */
typedef struct {
    int64_t M;
    int32_t N, K;
    fe_mat x, w, dout, pre;
    fe_mat dx, dw;
    void *dbias;
    fe_act act;
    void *work;
    int64_t work_bytes;
} fe_project_backward_args;
FE_API int64_t fe_project_backward_work(const fe_target *t, const fe_project_backward_args *a);
FE_API fe_status fe_project_backward(fe_target *t, const fe_project_backward_args *a, void *stream);

/* out [M, F] = act(x [M, K] w_gate [F, K]^T) * (x w_up [F, K]^T). gate_pre and up_pre: both or none of
 * the two products, float32 [M, F], which the gradient needs. Sizes as for fe_project. */
typedef struct {
    int64_t M;
    int32_t F, K;
    fe_mat x, w_gate, w_up, out, gate_pre, up_pre;
    fe_act act;
    void *work;
    int64_t work_bytes;
} fe_gated_ffn_args;
FE_API int64_t fe_gated_ffn_work(const fe_target *t, const fe_gated_ffn_args *a);
FE_API fe_status fe_gated_ffn(fe_target *t, const fe_gated_ffn_args *a, void *stream);

/* Gradients of fe_gated_ffn, for dh [M, F]: dout itself, or, with w_down [N, F], dout [M, N] w_down (the
 * gradient of a block h w_down^T, without a rounding in between). With dg = dh up act'(gate) and du =
 * dh act(gate) (gate, up: the two products as stored), rounded to the handle's type,
 *   dx [M, K] = dg w_gate + du w_up,  dw_gate [F, K] = dg^T x,  dw_up [F, K] = du^T x,
 *   dw_down [N, F] = dout^T h with h = act(gate) up, rounded as fe_gated_ffn's result;
 * each may be absent, the first two weights' both or none. */
typedef struct {
    int64_t M;
    int32_t F, K, N;
    fe_mat x, w_gate, w_up, w_down, dout, gate_pre, up_pre;
    fe_mat dx, dw_gate, dw_up, dw_down;
    fe_act act;
    void *work;
    int64_t work_bytes;
} fe_gated_ffn_backward_args;
FE_API int64_t fe_gated_ffn_backward_work(const fe_target *t, const fe_gated_ffn_backward_args *a);
FE_API fe_status fe_gated_ffn_backward(fe_target *t, const fe_gated_ffn_backward_args *a, void *stream);

/* With norm(v; w) = v / sqrt(mean(v^2) + eps) (w + offset) for rows v of d elements:
 *   y [R, d] = x + scale gate p,  p = norm(z; post_w) if post != 0, else z;
 *   n [R, d] = norm(y; pre_w), of y before it is rounded.
 *  z            the block's output; absent: y = x (post and gate must be absent too)
 *  post_w, pre_w  [d] or NULL: w + offset counts as 1
 *  gate         [ceil(R / gate_rows), d] or absent (1): row r of x takes row r / gate_rows, so that
 *               gate_rows is 1 for a gate of each row, the tokens of a sequence for a gate of each
 *               sequence, and R for a gate of each channel
 *  y, n         either may be absent; y may be x or z itself, n may be z itself (the same p and row)
 * scale and offset finite, eps finite and >= 0; R in 0..2^30, d in 1..2^20. */
typedef struct {
    int64_t R;
    int32_t d, post;
    fe_mat x, z, gate;
    int64_t gate_rows;
    const void *post_w, *pre_w;
    float scale, offset, eps;
    fe_mat y, n;
} fe_block_norm_args;
FE_API fe_status fe_block_norm(fe_target *t, const fe_block_norm_args *a, void *stream);

/* Gradients of fe_block_norm, for the outputs' gradients dy and dn [R, d] (either may be absent:
 * zero): dx, dz [R, d], dgate (as gate), dpost_w and dpre_w [d], each of which may be absent. The
 * other members are the forward call's. dx and dz may be dy or dn themselves (the same p and row). */
typedef struct {
    int64_t R;
    int32_t d, post;
    fe_mat x, z, gate;
    int64_t gate_rows;
    const void *post_w, *pre_w;
    float scale, offset, eps;
    fe_mat dy, dn, dx, dz, dgate;
    void *dpost_w, *dpre_w;
    void *work;
    int64_t work_bytes;
} fe_block_norm_backward_args;
FE_API int64_t fe_block_norm_backward_work(const fe_target *t, const fe_block_norm_backward_args *a);
FE_API fe_status fe_block_norm_backward(fe_target *t, const fe_block_norm_backward_args *a, void *stream);

/* With l = logits / temperature and log p = l - lse, lse = log sum_v exp(l_v), per row:
 *   logprob [R, J]      log p of tokens [R, J] (device int32); a negative token is none: 0
 *   entropy [R]         - sum_v p_v log p_v (terms with p = 0 count as 0)
 *   lse [R]
 *   stats [R, 2]        the row's largest logit m and log sum_v exp((logit_v - m) / temperature), for the
 *                       gradient (a row without tokens: -inf as the second)
 *   top_id, top_logprob [R, K]  the K largest logits, descending, equal ones by the smaller index, and
 *                       their log p
 *  logits   [R, V] of `dtype` (FE_F32 or FE_BF16, whatever the handle's)
 *  J 0..64, K 0..32, K <= V; logprob and tokens may be NULL for J = 0, top_id and top_logprob for
 *  K = 0; entropy, lse and stats may be NULL. temperature from 2^-64 to 2^64. V in 1..2^30.
 * Ruled-out tokens are logits of minus infinity. A row that has nothing else gets lse and every log p
 * = -inf and entropy 0; a row with NaN or +inf gets NaN for all of them (and NaN comes first among
 * the largest logits). A token >= V sets FE_ERR_DEVICE and counts as none. */
typedef struct {
    int64_t R;
    int32_t V, J, K;
    fe_mat logits;
    fe_dtype dtype;
    float temperature;
    const int32_t *tokens;
    float *logprob, *entropy, *lse, *stats;
    int32_t *top_id;
    float *top_logprob;
} fe_token_logprobs_args;
FE_API fe_status fe_token_logprobs(fe_target *t, const fe_token_logprobs_args *a, void *stream);

/* Gradient of fe_token_logprobs: dlogits [R, V] of the logits' type, which may be the logits
 * themselves (the same p and row), for the gradients dlogprob [R, J], dentropy [R], dlse [R] and
 * dtop_logprob [R, K] (each NULL: zero). stats is the forward call's, entropy too (needed for
 * dentropy), top_id for dtop_logprob (entries outside [0, V) are none). The same token twice adds up.
 * A row that has only ruled-out tokens gets zeros but for what its tokens' own gradients say. */
typedef struct {
    int64_t R;
    int32_t V, J, K;
    fe_mat logits;
    fe_dtype dtype;
    float temperature;
    const int32_t *tokens, *top_id;
    const float *stats, *entropy, *dlogprob, *dentropy, *dlse, *dtop_logprob;
    fe_mat dlogits;
} fe_token_logprobs_backward_args;
FE_API fe_status fe_token_logprobs_backward(fe_target *t, const fe_token_logprobs_backward_args *a, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FE_LAYER_H */
