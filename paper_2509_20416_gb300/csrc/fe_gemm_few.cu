// Matrix products of few rows of bfloat16 (single tokens, a tree's nodes): bound by the weights' bytes.
//
// The weights take the side of the tensor cores' 128 rows, so that every byte of them is copied once by
// TMA and 16 to 128 tokens are the columns: D [128 weight rows, NT tokens] in tensor memory. A cluster of
// 1 to 8 CTAs shares a block of 128 rows and divides the summed index; the parts are added in
// their order through distributed shared memory, each CTA finishing its share of the tokens. A gated
// pair's block is 64 rows of either matrix.
//
// Measured (GB300): one token through a gated pair of 14336 x 4096 38 to 40 us (86 to 90 % of the copy rate; 109 us
// as tiles of 256 rows), 71 rows through 28672 x 8192 151 us (92 %), 49 rows to 128256 172 us (91 %), one token
// through 6144 x 4096 13.4 us, where a CTA's start, its first copies and the join are half. The first copies
// go out before tensor memory is allocated.
#include "fe_gemm_plan.h"
#include "fe_gemm_tc.cuh"
#include "fe_tensor_map.h"

namespace fe {

namespace {

constexpr int kFewThreads = 128;

struct FewBarriers {
    uint64_t full[kFewStages], empty[kFewStages], done;
    uint32_t tmem;
};

__global__ void __launch_bounds__(kFewThreads)
    gemm_few_kernel(const __grid_constant__ GemmArgs g, const __grid_constant__ CUtensorMap wmap0, const __grid_constant__ CUtensorMap wmap1,
                    const __grid_constant__ CUtensorMap xmap, const __grid_constant__ FewArgs f) {
    extern __shared__ unsigned char raw[];
    unsigned char* const ring = (unsigned char*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    __shared__ FewBarriers bar;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const bool gated = g.e.kind == FINISH_GATED;
    const int rank = f.ranks > 1 ? (int)cluster_rank() : 0;
    const int64_t block = blockIdx.x / f.ranks;
    const int n0 = (int)block * (gated ? 64 : 128);
    const int slices = (g.K + 63) / 64;
    const int k0 = (int)((int64_t)slices * rank / f.ranks), k1 = (int)((int64_t)slices * (rank + 1) / f.ranks);
    int cols = 32;
    while (cols < f.nt) cols *= 2;

    const auto copy = [&](int k, int slot) {
        unsigned char* const w = ring + slot * f.stage_bytes;
        mbar_arrive_expect_tx(&bar.full[slot], 16384 + f.nt * 128);
        tma_box(w, &wmap0, k * 64, n0, &bar.full[slot]);
        if (gated) tma_box(w + 8192, &wmap1, k * 64, n0, &bar.full[slot]);
        tma_box(w + 16384, &xmap, k * 64, 0, &bar.full[slot]);
    };
    const int ahead = min(f.stages, k1 - k0);
    if (warp == 0 && lane == 0) {
        for (int i = 0; i < f.stages; ++i) {
            mbar_init(&bar.full[i], 1);
            mbar_init(&bar.empty[i], 1);
        }
        mbar_init(&bar.done, 1);
        mbar_fence_init();
        for (int i = 0; i < ahead; ++i) copy(k0 + i, i);  // (before the CTA is set up)
    }
    if (warp == 1) tc_alloc(&bar.tmem, cols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bar.tmem;

    if (warp == 0) {  // ---- copies
        if (lane == 0) {
            int slot = ahead == f.stages ? 0 : ahead, n = ahead;
            uint32_t phase = 0;  // of the slot's use before
            bool ok = true;
            for (int k = k0 + ahead; k < k1; ++k, ++n) {
                if (!(ok = mbar_wait(&bar.empty[slot], phase, g.status))) break;
                copy(k, slot);
                if (++slot == f.stages) slot = 0, phase ^= 1;
            }
            if (!ok) {  // (what is in flight lands before the CTA ends)
                for (int i = n > f.stages ? n - f.stages : 0; i < n; ++i)
                    mbar_wait(&bar.full[i % f.stages], (uint32_t)(i / f.stages) & 1, g.status, 50000000LL);
            }
        }
        __syncwarp();
    } else if (warp == 1) {  // ---- products
        if (one_lane()) {
            const uint32_t id = idesc_bf16_f32(kFewRows, f.nt);
            int slot = 0;
            uint32_t phase = 0;
            for (int k = k0; k < k1; ++k) {
                if (!mbar_wait(&bar.full[slot], phase, g.status)) {
                    for (int i = 1; i < f.stages && k + i < k1; ++i) {  // (the copies behind it land before the CTA ends)
                        const int s = slot + i < f.stages ? slot + i : slot + i - f.stages;
                        mbar_wait(&bar.full[s], slot + i < f.stages ? phase : phase ^ 1, g.status, 50000000LL);
                    }
                    break;
                }
                tc_fence_after();
                const uint32_t at = smem_u32(ring + slot * f.stage_bytes);
                const uint64_t wd = sw128_desc(at), xd = sw128_desc(at + 16384);
#pragma unroll
                for (int i = 0; i < 4; ++i) tc_mma(tmem, wd + 2 * i, xd + 2 * i, id, k > k0 || i > 0);
                tc_commit(&bar.empty[slot]);
                if (++slot == f.stages) slot = 0, phase ^= 1;
            }
            tc_commit(&bar.done);
        }
        __syncwarp();
    }
    // ---- a CTA's sums, by token, in the ring's place
    const bool ok = mbar_wait(&bar.done, 0, g.status);
    __syncthreads();  // (the copying lane has seen its copies land, or given up)
    tc_fence_after();
    float* const part = (float*)ring;
    const int M = (int)g.M;
    for (int c = 0; c < f.nt; c += 16) {
        float z[16];
        tc_ld16(tmem + ((uint32_t)(warp * 32) << 16) + c, z);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (c + i < M) part[(c + i) * kPartRow + threadIdx.x] = ok && k1 > k0 ? z[i] : 0.f;
        }
    }
    tc_fence_before();
    if (f.ranks > 1) cluster_sync_all();
    else __syncthreads();
    if (warp == 1) tc_dealloc(tmem, cols);
    // ---- the cluster's, for this CTA's tokens
    const Finish& e = g.e;
    uint32_t base[kFewMost];
#pragma unroll
    for (int r = 0; r < kFewMost; ++r) base[r] = r < f.ranks ? peer_u32(part, r) : 0;
    const auto total = [&](int token, int row) {
        if (f.ranks == 1) return part[token * kPartRow + row];
        const uint32_t off = (token * kPartRow + row) * 4;
        float v[kFewMost];
#pragma unroll
        for (int r = 0; r < kFewMost; ++r) v[r] = r < f.ranks ? load_peer(base[r] + off) : 0.f;
        float s = v[0];
#pragma unroll
        for (int r = 1; r < kFewMost; ++r) s += v[r];
        return s;
    };
    if (gated) {
        const int row = threadIdx.x % 64, n = n0 + row;
        for (int t = rank + f.ranks * (threadIdx.x / 64); t < M && n < g.N; t += 2 * f.ranks) {
            const float z = total(t, row), u = total(t, 64 + row);
            if (e.pre) {
                e.pre[t * e.pre_row + n] = z;
                e.pre2[t * e.pre2_row + n] = u;
            }
            store_one((bf16_t*)e.out + t * e.out_row + n, act_value<true>(e.act, z) * u);
        }
    } else {
        const int row = threadIdx.x, n = n0 + row;
        const float b = e.bias && n < g.N ? load_one((const bf16_t*)e.bias + n) : 0.f;
        for (int t = rank; t < M && n < g.N; t += f.ranks) {
            float z = total(t, row) + b;
            if (e.pre) e.pre[t * e.pre_row + n] = z;
            if (e.act != FE_ACT_NONE) z = act_value<true>(e.act, z);
            if (e.res) z += load_one((const bf16_t*)e.res + t * e.res_row + n);
            store_one((bf16_t*)e.out + t * e.out_row + n, z);
        }
    }
    if (f.ranks > 1) cluster_sync_all();  // (the others have read this CTA's sums)
}

}  // namespace

cudaError_t gemm_few_prepare() {
    return cudaFuncSetAttribute(gemm_few_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem);
}

bool gemm_few_takes(const GemmArgs& g) {
    return g.M <= 128 && !g.a_t && !g.b_t && g.segs == 1 && !g.twice && (g.e.kind == FINISH_PLAIN || g.e.kind == FINISH_GATED);
}

cudaError_t launch_gemm_few(const GemmArgs& g, int num_sms, cudaStream_t st) {
    const bool gated = g.e.kind == FINISH_GATED;
    const int rows = gated ? 64 : 128;
    const int64_t blocks = ((int64_t)g.N + rows - 1) / rows;
    int smem = 0;
    const FewArgs f = few_plan(g.M, g.N, g.K, gated, num_sms, &smem);
    CUtensorMap w0, w1, x;
    const auto map = [](CUtensorMap* m, const fe_mat& a, int64_t r, int64_t c, int box_rows) { return tensor_map_bf16(m, a, r, c, box_rows); };
    if (!map(&w0, g.b[0], g.N, g.K, rows) || !map(&w1, g.b[gated ? 1 : 0], g.N, g.K, rows) || !map(&x, g.a[0], g.M, g.K, f.nt)) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(blocks * f.ranks));
    cfg.blockDim = dim3(kFewThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = f.ranks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, gemm_few_kernel, g, w0, w1, x, f);
}

}  // namespace fe
