/*
 * fe_target.h -- C ABI of the target-side operators of a verification cycle (Sec. 2.4,
 * "Parallel Verification" and "Update and Iterate"): what a layer of the target model needs
 * around its own matrices to score a draft tree on a GB300 (sm_103a).
 *
 *   fe_rope            rotary positions on queries and keys, and their gradient
 *   fe_cache_write     key/value rows into a layer's cache, rotated and quantised on the way
 *   fe_cache_read      cache rows back as dense rows
 *   fe_tree_attention  attention of a tree's nodes (or of consecutive tokens) over the cache
 *   fe_cache_keep      the accepted nodes' rows moved to their final slots, all layers at once
 *
 * A cycle: fe_build_tree's T nodes of sequence b take cache slots P_b .. P_b + T - 1 in node
 * order, while their positions are P_b + depth (fe_verify_greedy's pos_ids). In each layer the
 * nodes' rows are written with fe_cache_write, then fe_tree_attention lets node i see the
 * prefix and its ancestors. After fe_verify_greedy or fe_verify_sampled, fe_cache_keep moves
 * the accepted path's rows next to the prefix, and the next cycle starts at P_b + 1 + n_accept.
 *
 * The conventions of fe_draft.h hold: status codes, device and host pointers, streams,
 * asynchronous calls with host-side argument checks, device-side range errors in a status word
 * (fe_target_status) with the offending work skipped, one handle not used from two streams at
 * once, no exceptions. Strides count elements of the tensor's type; the innermost dimension
 * (head_dim) is contiguous. Rows and strides need no alignment beyond the type's own; 16-byte
 * aligned ones are faster. Cache buffers start on a 16-byte boundary.
 */
#ifndef FE_TARGET_H
#define FE_TARGET_H

#include "fe_draft.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Which elements of a head a rotation pairs: HALF pairs (i, i + rope_dim / 2), INTERLEAVED
 * pairs (2 i, 2 i + 1); pair i turns by pos * f_i. Elements from rope_dim on pass through. */
typedef enum { FE_ROPE_HALF = 0, FE_ROPE_INTERLEAVED = 1 } fe_rope_layout;

/* Frequencies for long contexts, with b_i = theta^(-2 i / rope_dim), s = rope_factor,
 * L = rope_orig (the context the model was first trained on):
 *   NONE    f_i = b_i
 *   LINEAR  f_i = b_i / s (positions squeezed)
 *   NTK     f_i = (theta s^(rope_dim / (rope_dim - 2)))^(-2 i / rope_dim) (rope_dim > 2)
 *   BANDS   by turns per context t_i = L b_i / 2 pi, w = clamp((t_i - low) / (high - low), 0, 1):
 *           f_i = b_i ((1 - w) / s + w)          (LLaMA 3.1's rule; low 1, high 4, L 8192)
 *   YARN    dim(r) = rope_dim ln(L / (2 pi r)) / (2 ln theta); lo = max(floor(dim(low)), 0),
 *           hi = min(ceil(dim(high)), rope_dim - 1), w = clamp((i - lo) / max(hi - lo, 0.001), 0, 1):
 *           f_i = b_i (w / s + 1 - w), cos and sin times 0.1 ln s + 1 (low 32, high 1)
 * with low = rope_low and high = rope_high. */
typedef enum {
    FE_ROPE_NONE = 0,
    FE_ROPE_LINEAR = 1,
    FE_ROPE_NTK = 2,
    FE_ROPE_BANDS = 3,
    FE_ROPE_YARN = 4
} fe_rope_scaling;

/* Attention shape of the target's layers and of their caches. */
typedef struct {
    int32_t n_heads;     /* query heads H */
    int32_t n_kv_heads;  /* key/value heads Hkv, a divisor of H */
    int32_t head_dim;    /* hd: 64 or 128 */
    int32_t max_batch;   /* sequences of a call; rows of a contiguous cache. 1..65535 */
    int32_t max_seq;     /* cache slots per sequence; positions lie in [0, max_seq). At most 2^28 */
    int32_t page_size;   /* 0: contiguous caches; > 0: rows per page (any size) */
    fe_dtype dtype;      /* FE_F32 or FE_BF16: q, k, v and output rows */
    fe_dtype cache_dtype; /* dtype, or FE_E4M3 with FE_BF16 rows */
    int32_t rope_dim;    /* rotated elements of a head: even, 2..head_dim */
    fe_rope_layout rope_layout;
    fe_rope_scaling rope_scaling;
    float rope_theta;    /* > 1 */
    float rope_factor;   /* s >= 1 (all but NONE) */
    float rope_low, rope_high; /* BANDS: 0 < low < high; YARN: low > high > 0 */
    float rope_orig;     /* L >= 1 (BANDS and YARN) */
} fe_target_config;

typedef struct fe_target fe_target;

/* A handle on the current device. It holds the rotation table (max_seq x rope_dim / 2 cosines
 * and sines, computed in double precision, stored in float32) and the attention's workspace; it
 * holds no cache. Orders its own work on `stream` and synchronises it. */
FE_API fe_status fe_target_init(const fe_target_config *cfg, void *stream, fe_target **out);

/* Release the handle (synchronises its device first). NULL is a no-op. */
FE_API void fe_target_free(fe_target *t);

/* Synchronise `stream`, return and clear the handle's device status word: FE_OK,
 * FE_ERR_CAPACITY (a slot or position outside [0, max_seq)), FE_ERR_DEVICE (a page id, row
 * count or path out of range) or FE_ERR_TIMEOUT. */
FE_API fe_status fe_target_status(fe_target *t, void *stream);

/* Rows of a [B, T, heads, hd] tensor with strides in elements. */
typedef struct {
    void *p;
    int64_t batch, token, head;
} fe_rows;

/* One layer's cache:
 *   k, v              page_size == 0: [max_batch, Hkv, max_seq, hd]; else a pool
 *                     [n_pages, Hkv, page_size, hd], as in fe_draft.h, of the cache type
 *   k_scale, v_scale  FE_E4M3 only: float32 [max_batch, Hkv, max_seq] or
 *                     [n_pages, Hkv, page_size]; a row stands for its e4m3 numbers times its
 *                     scale, a power of two from 2^-120 to 2^120 (as fe_cache_write stores them;
 *                     in slots that no node sees anything, as in the rows themselves),
 *                     so every value is a bfloat16 number */
typedef struct {
    void *k, *v;
    float *k_scale, *v_scale;
} fe_kv;

/* Page table of a call, device [B, ceil(max_seq / page_size)] int32 (paged caches only). */
typedef struct {
    const int32_t *table;
    int32_t n_pages;
} fe_pages;

/* Rotary positions. q [B, T, H, hd] and k [B, T, Hkv, hd] (either may have p == NULL) are
 * rotated to pos (device [B, T] int32) and written to q_out and k_out, which may be the inputs
 * themselves (the same pointer and strides) but must not overlap them otherwise. The rotation
 * is computed in float32 and rounded once. backward != 0 computes the gradient instead: with
 * the outputs' gradients as q and k, each pair turns back (and keeps YARN's factor), the
 * transpose of the forward map. A row with a position outside [0, max_seq) is left unwritten
 * and sets FE_ERR_CAPACITY. B in 1..max_batch, T >= 1. */
typedef struct {
    int32_t B, T;
    fe_rows q, k, q_out, k_out;
    const int32_t *pos;
    int32_t backward;
} fe_rope_args;
FE_API fe_status fe_rope(fe_target *t, const fe_rope_args *a, void *stream);

/* Key/value rows into a cache: row i < n_rows[b] of sequence b goes to slot start[b] + i.
 *  k, v      [B, T, Hkv, hd] rows of the handle's type
 *  pos       device [B, T] int32 or NULL. With pos the keys are rotated to it first (in
 *            float32: an FE_E4M3 cache rounds once), and, when q.p is set, q [B, T, H, hd] is
 *            rotated into q_out as by fe_rope (all T rows). Without pos the keys are stored as
 *            they are and q must be NULL.
 *  start     device [B] int32; n_rows device [B] int32 in 0..T, or NULL for T. Rows from n_rows[b]
 *            on are not looked at, their positions only for q
 * FE_E4M3: each row of a head gets the scale 2^c with the smallest c >= -120 for which no
 * finite element exceeds 448 times it, and each element / 2^c is rounded to e4m3 (ties to
 * even); a NaN or infinite element is stored as e4m3's NaN. Rows whose slot lies outside
 * [0, max_seq), whose page id is outside [0, n_pages) or whose position is out of range are
 * skipped and reported by fe_target_status. Two rows of a call must not share a slot. */
typedef struct {
    int32_t B, T;
    fe_rows k, v, q, q_out;
    const int32_t *pos, *start, *n_rows;
    fe_kv cache;
    fe_pages pages;
} fe_cache_write_args;
FE_API fe_status fe_cache_write(fe_target *t, const fe_cache_write_args *a, void *stream);

/* Cache rows as dense rows of the handle's type: row i < n_rows[b] of k_out, v_out
 * [B, L, Hkv, hd] is slot start[b] + i; rows from n_rows[b] on are set to zero, and so is a row
 * whose slot or page is out of range (reported by fe_target_status). */
typedef struct {
    int32_t B, L;
    const int32_t *start, *n_rows;
    fe_kv cache;
    fe_pages pages;
    fe_rows k_out, v_out;
} fe_cache_read_args;
FE_API fe_status fe_cache_read(fe_target *t, const fe_cache_read_args *a, void *stream);

/* Attention over the cache (all keys and values, the nodes' own among them, are in it):
 *   node i of sequence b sees slot s < P_b, and slot P_b + c for the nodes c < n_b with
 *   mask[b][i][c] != 0 (mask == NULL: c <= i, consecutive tokens);
 *   out[b][i][h] = sum_s softmax_s(scale q[b][i][h] . K[s]) V[s], over h's shared KV head
 *   h / (H / Hkv); lse[b][i][h] = log sum_s exp(scale q . K[s]).
 *  q, out      [B, T, H, hd] of the handle's type; out must not overlap q
 *  lse         device [B, T, H] float32 or NULL
 *  prefix_len  device [B] int32: P_b >= 0, P_b + n_b <= max_seq
 *  n_nodes     device [B] int32 in 0..T, or NULL for T
 *  mask        device [B, T, T] uint8 (fe_build_tree's mask) or NULL
 *  scale       finite, > 0
 * Softmax statistics and sums are float32. FE_BF16 handles round the probabilities to bfloat16 (up
 * to 2^-8 of each) for the product with the values. Over an FE_E4M3 cache they take a query
 * element exactly from 2^-9 of its row's largest on and to 2^-17 of the largest below that, and a
 * row with a non-finite element as NaN. An FE_F32 handle keeps 32 bits throughout. A node that
 * sees no slot, or only scores of minus infinity, and every node i >= n_b get a zero row and lse =
 * -inf; slots that a node does not see do not affect it whatever they hold, NaN included. A
 * sequence with P_b or n_b out of range counts as n_b = 0 and sets FE_ERR_CAPACITY; a bad page id
 * sets FE_ERR_DEVICE and its rows count as zeros. The result does not depend on timing: the same
 * call gives the same bits.
 * B in 1..max_batch, T >= 1. FE_ERR_UNSUPPORTED for a shape whose work could pass 2^31 units, of 64
 * rows x 64 slots (float32) or 128 x 128 (where slots are nodes' a half more, over bfloat16). */
typedef struct {
    int32_t B, T;
    fe_rows q, out;
    float *lse;
    const int32_t *prefix_len, *n_nodes;
    const uint8_t *mask;
    float scale;
    fe_kv cache;
    fe_pages pages;
} fe_tree_attention_args;
FE_API fe_status fe_tree_attention(fe_target *t, const fe_tree_attention_args *a, void *stream);

/* Accepted rows to their final slots, in n_layers caches (host array) of one page table: for
 * each sequence b and j < n_accept[b], the rows of slot start[b] + path[b][j] become those of
 * slot start[b] + 1 + j (the root's row stays at slot start[b]), as stored, scales included.
 *  path      device [B, N] int32: the accepted nodes in order, strictly increasing, >= 1
 *            (fe_verify_greedy's and fe_verify_sampled's path); entries from n_accept[b] on
 *            are ignored
 *  n_accept  device [B] int32 in 0..N
 * A sequence with a path, count, slot or page out of range is skipped and reported by
 * fe_target_status. */
typedef struct {
    int32_t B, N, n_layers;
    const int32_t *path, *n_accept, *start;
    const fe_kv *caches;
    fe_pages pages;
} fe_cache_keep_args;
FE_API fe_status fe_cache_keep(fe_target *t, const fe_cache_keep_args *a, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FE_TARGET_H */
