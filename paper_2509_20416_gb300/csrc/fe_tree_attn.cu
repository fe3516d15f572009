// Attention of a draft tree's nodes (or of consecutive tokens) over the cache
// (fe_tree_attention): the variants and their launches.
#include "fe_tensor_map.h"
#include "fe_tree_attn_join.cuh"
#include "fe_tree_attn_simt.cuh"
#include "fe_tree_attn_tc.cuh"

namespace fe {

namespace {

template <typename QT, int HD, int ROWS>
cudaError_t launch_join(const TreeAttnArgs& a, int ncta, cudaStream_t st) {
    const int rows = (int)min((int64_t)a.T * a.G, (int64_t)ROWS);  // of an item
    return launch_k(tree_attn_join_kernel<QT, HD, ROWS>, dim3(ncta, ((rows + 31) / 32 * (HD / 16) + kJoinWarps - 1) / kJoinWarps), dim3(kJoinThreads), 0, st, true, a);
}

template <int HD, int NI>
cudaError_t launch_simt(const TreeAttnArgs& args, int num_sms, cudaStream_t st) {
    using SM = SimtSmem<HD, NI>;
    static_assert(SM::kCtas * 64 <= kAttnItemRows && SM::kCtas <= kAttnCtasPerSm, "the workspace's rows and notes");
    TreeAttnArgs a = args;
    a.part_rows = 64;
    const int grid = num_sms * SM::kCtas;
    const cudaError_t e = launch_k(tree_attn_simt_kernel<HD, NI>, dim3(grid), dim3(kSimtThreads), sizeof(SM), st, false, a);
    if (e != cudaSuccess) return e;
    return launch_join<float, HD, 16 * NI>(a, grid, st);
}

// Rows of a TMA box: a bfloat16 cache's tiles of 128 slots come in boxes that lie inside one page
// and fill whole 8-row swizzle groups; 0 where no such box exists or is worth it (pages of other
// sizes, caches of less than a tile), and the loaders' copies do it all. The TMA unit takes some 110
// to 150 clocks a box: 32 sequences of 17 nodes over pages of 8 took 123 us by TMA and 83 without,
// pages of 16 88 us by TMA, 83 without and 74 when it brings the keys and the loaders the values.
int tma_box_rows(const CacheView& c, int groups) {
    if (groups <= 0) return 0;
    if (c.page_size == 0) return c.max_seq >= kTcTile ? kTcTile : 0;
    int b = kTcTile;
    while (c.page_size % b) b /= 2;
    return b >= 16 ? b : 0;
}

// The cache as [groups][rows][hd], rows of a page or sequence, groups = (pages or sequences) x
// heads; boxes of 64 bfloat16 or hd e4m3 elements, swizzled over their bytes
bool make_map(CUtensorMap* map, const void* base, bool e4m3, int hd, int rows, int groups, int box_rows) {
    const cuuint64_t es = e4m3 ? 1 : 2;
    const cuuint64_t dims[3] = {(cuuint64_t)hd, (cuuint64_t)rows, (cuuint64_t)groups};
    const cuuint64_t strides[2] = {(cuuint64_t)hd * es, (cuuint64_t)rows * hd * es};
    const cuuint32_t box[3] = {e4m3 ? (cuuint32_t)hd : 64u, (cuuint32_t)box_rows, 1}, step[3] = {1, 1, 1};
    const EncodeTiled encode = encode_tiled();
    return encode && encode(map, e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3,
                            const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            box[0] * es == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The queries as [B][T][H][hd]; a block of 128 rows is a box of G heads and 128 / G nodes, where G
// is a power of two and the strides are what a map can hold (whole 16 bytes, as they mostly are).
bool make_q_map(CUtensorMap* map, const TreeAttnArgs& a, int hd) {
    if (!a.q_vec || a.G > 128 || 128 % a.G) return false;
    cuuint64_t strides[3] = {(cuuint64_t)a.q.head * 2, (cuuint64_t)a.q.token * 2, (cuuint64_t)a.q.batch * 2};
    const cuuint64_t dims[4] = {(cuuint64_t)hd, (cuuint64_t)a.H, (cuuint64_t)a.T, (cuuint64_t)a.B};
    for (int i = 0; i < 3; ++i) {
        if (dims[i + 1] == 1) strides[i] = (cuuint64_t)hd * 2;  // (an extent of 1: the stride is not used)
        if ((int64_t)strides[i] <= 0 || strides[i] >= (cuuint64_t)1 << 40) return false;
    }
    const cuuint32_t box[4] = {64, (cuuint32_t)a.G, (cuuint32_t)(128 / a.G), 1}, step[4] = {1, 1, 1, 1};
    const EncodeTiled encode = encode_tiled();
    return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, a.q.p, dims, strides, box, step,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD, bool Q8, int MT>
cudaError_t launch_tc(const TreeAttnArgs& args, int num_sms, cudaStream_t st) {
    TreeAttnArgs a = args;
    a.part_rows = kAttnItemRows;
    CUtensorMap kmap{}, vmap{}, qmap{};
    a.q_tma = make_q_map(&qmap, a, HD);
    const CacheView& c = a.cache;
    const int64_t groups = (int64_t)(c.page_size ? c.n_pages : a.B) * a.Hkv;
    a.box_rows = tma_box_rows(c, groups < 0x7FFFFFFF ? (int)groups : 0);
    const int rows = c.page_size ? c.page_size : c.max_seq;
    if (a.box_rows && !(make_map(&kmap, c.k, Q8, HD, rows, (int)groups, a.box_rows) &&
                        (Q8 || make_map(&vmap, c.v, false, HD, rows, (int)groups, a.box_rows))))
        return cudaErrorInvalidValue;
    const cudaError_t e = launch_k(tree_attn_tc_kernel<HD, Q8, MT>, dim3(num_sms), dim3(TcShape<HD, Q8, MT>::kThreads),
                                   tc_smem<HD, Q8, MT>(), st, false, a, kmap, vmap, qmap);
    if (e != cudaSuccess) return e;
    return launch_join<bf16_t, HD, kAttnItemRows>(a, num_sms, st);
}

template <typename K>
cudaError_t allow_smem(K kern, size_t bytes) {
    return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <int HD>
cudaError_t prepare() {
    cudaError_t e;
    if ((e = allow_smem(tree_attn_simt_kernel<HD, 1>, sizeof(SimtSmem<HD, 1>))) != cudaSuccess) return e;
    if ((e = allow_smem(tree_attn_simt_kernel<HD, 2>, sizeof(SimtSmem<HD, 2>))) != cudaSuccess) return e;
    if ((e = allow_smem(tree_attn_simt_kernel<HD, 4>, sizeof(SimtSmem<HD, 4>))) != cudaSuccess) return e;
    if ((e = allow_smem(tree_attn_tc_kernel<HD, false, 1>, tc_smem<HD, false, 1>())) != cudaSuccess) return e;
    if ((e = allow_smem(tree_attn_tc_kernel<HD, false, 2>, tc_smem<HD, false, 2>())) != cudaSuccess) return e;
    if ((e = allow_smem(tree_attn_tc_kernel<HD, true, 1>, tc_smem<HD, true, 1>())) != cudaSuccess) return e;
    return allow_smem(tree_attn_tc_kernel<HD, true, 2>, tc_smem<HD, true, 2>());
}

template <int HD>
cudaError_t launch_hd(const TreeAttnArgs& a, fe_dtype dtype, fe_dtype cache_dtype, int num_sms, cudaStream_t st) {
    const int64_t rows = (int64_t)a.T * a.G;
    if (dtype == FE_F32)
        return rows <= 16   ? launch_simt<HD, 1>(a, num_sms, st)
               : rows <= 32 ? launch_simt<HD, 2>(a, num_sms, st)
                            : launch_simt<HD, 4>(a, num_sms, st);
    const bool one = rows <= 128;  // every item fits one 128-row block: more tiles in flight
    if (cache_dtype == FE_E4M3)
        return one ? launch_tc<HD, true, 1>(a, num_sms, st) : launch_tc<HD, true, 2>(a, num_sms, st);
    return one ? launch_tc<HD, false, 1>(a, num_sms, st) : launch_tc<HD, false, 2>(a, num_sms, st);
}

}  // namespace

cudaError_t tree_attn_prepare() {
    const cudaError_t e = prepare<64>();
    return e != cudaSuccess ? e : prepare<128>();
}

bool tree_attn_fits(const TreeAttnArgs& a, fe_dtype dtype, fe_dtype cache_dtype) {
    return attn_plan_fits(dtype, cache_dtype, a.B, a.Hkv, a.T, a.G, a.cache.max_seq);
}

cudaError_t launch_tree_attn(const TreeAttnArgs& a, fe_dtype dtype, fe_dtype cache_dtype, int hd, int num_sms,
                             cudaStream_t st) {
    return hd == 128 ? launch_hd<128>(a, dtype, cache_dtype, num_sms, st) : launch_hd<64>(a, dtype, cache_dtype, num_sms, st);
}

}  // namespace fe
