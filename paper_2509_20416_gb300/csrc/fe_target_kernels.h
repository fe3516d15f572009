// Internal launch interface of the target-side operators (include/fe_target.h).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "fe_kernels.h"
#include "fe_target.h"

namespace fe {

// Where a layer's cache rows lie. Row index (of head_dim elements, and of the scales) of
// slot s of sequence b and head h: (b Hkv + h) max_seq + s, or, paged,
// (table[b max_pages + s / page_size] Hkv + h) page_size + s % page_size.
struct CacheView {
    void *k, *v;
    float *ks, *vs;
    const int* table;
    int n_pages, page_size, max_pages, max_seq, Hkv;
};

// rotation of rows: the table holds (cos, sin) [max_seq][rope_dim / 2]
struct RopeView {
    const float2* table;
    int dim, interleaved, max_pos;
};

// fe_rope (cache_kind 0) and fe_cache_write (1: cache of the rows' type, 2: e4m3)
struct RowsArgs {
    int B, T, HA, HB;  // HA heads of rotated rows a; HB heads of rows b (fe_rope's k), or KV heads
    fe_rows a_in, a_out, b_in, b_out;  // b_in: fe_rope's k or fe_cache_write's k
    fe_rows v_in;
    const int *pos, *start, *n_rows;
    RopeView rope;
    float dir;  // +1 forward, -1 the gradient: the sign of the sines
    CacheView cache;
    int* status;
};

struct ReadArgs {
    int B, L;
    const int *start, *n_rows;
    CacheView cache;
    fe_rows k_out, v_out;
    int* status;
};

constexpr int kKeepMaxLayers = 128;  // per launch (the pointers travel as kernel arguments)

struct KeepArgs {
    int B, N, n_layers, row_bytes, layers_per_warp;
    const int *path, *n_accept, *start;
    CacheView cache;  // (its pointers are per layer, below)
    fe_kv layer[kKeepMaxLayers];
    int* status;
};

// What an attention CTA leaves for the join of split items: the item that it begins and that goes
// on to CTA `last` (-1: none), and whether it holds a share of an item begun before it.
struct SplitDesc {
    int b, h, m, rows, last, has0, pad[2];
};

struct TreeAttnArgs {
    int B, T, H, Hkv, G;
    fe_rows q, out;
    float* lse;
    const int *prefix, *nodes;
    const uint8_t* mask;
    float scale;
    CacheView cache;
    SplitDesc* split;         // [G], of every attention CTA
    int part_rows;            // rows of a partial item in the workspace: per CTA two items,
    float *part_o, *part_ml;  // sums [2 G][hd / 4][part_rows][4], (max, sum) [2 G][part_rows][2]
    int* status;
    int q_vec, out_vec;  // rows of q / out on 16-byte boundaries (out: 2 on 32-byte ones)
    int box_rows;        // cache rows of a TMA box (0: no tensor maps)
    int q_tma;           // the queries come by TMA too
};

// rows of an attention item whose partial results the workspace holds, per CTA and slot
constexpr int kAttnItemRows = 256;
constexpr int kAttnCtasPerSm = 2;  // at most (with items of at most 128 rows each then)

cudaError_t launch_rope_table(float2* table, int max_seq, int pairs, const double* inv_freq, double amplitude,
                              int num_sms, cudaStream_t st);
cudaError_t launch_rows(const RowsArgs& a, fe_dtype dtype, int hd, int cache_kind, cudaStream_t st);
cudaError_t launch_cache_read(const ReadArgs& a, fe_dtype dtype, fe_dtype cache_dtype, int hd, cudaStream_t st);
cudaError_t launch_cache_keep(const KeepArgs& a, int num_sms, cudaStream_t st);
cudaError_t tree_attn_prepare();
// whether the schedule can count the work of every call of this shape
bool tree_attn_fits(const TreeAttnArgs& a, fe_dtype dtype, fe_dtype cache_dtype);
cudaError_t launch_tree_attn(const TreeAttnArgs& a, fe_dtype dtype, fe_dtype cache_dtype, int hd, int num_sms,
                             cudaStream_t st);

}  // namespace fe
