// Matrix products of bfloat16 on the tensor cores (fe_layer.h's products and their gradients): C = A B^T
// with either operand stored by rows or by its summed index, float32 sums in tensor memory.
//
// Persistent pairs of CTAs (cta_group::2) make tiles of 256 x BN: each CTA brings, by TMA, 128 rows of A
// and BN / 2 of B in slices of 64 of the summed index, so that an SM reads half of what a CTA of its own
// would for the same products. Warp 0 copies, warp 1 of the first CTA issues the products, warps 2 to 5
// finish a tile (bias, activation, residual, gate, rounding) while the next one is summed in the
// other half of tensor memory. The MN-major operand forms spare the gradients every transpose:
// dx = dz w reads w by columns, dw = dz^T x both operands.
#include "fe_gemm_tc.cuh"
#include "fe_tensor_map.h"

namespace fe {

namespace {

constexpr int kTcThreads = 192;
constexpr int kTileM = 256, kSliceK = 64;

template <int BN>
struct TcTile {
    static constexpr int kA = 128 * kSliceK * 2, kB = BN / 2 * kSliceK * 2;
    static constexpr int kStages = BN == 256 ? 6 : 8;
    static constexpr int kRing = kStages * (kA + kB);
    static constexpr int kTmem = 2 * BN;  // two accumulators
    static constexpr int kSmem = kRing + 1024 /* alignment */ + 512;
};

struct TcBarriers {
    uint64_t full[8], empty[8], done[2], free[2], drain;
    uint32_t tmem;
};

struct TcMaps {
    CUtensorMap a[2], b[2];
};

// which tile comes where: supergroups of 8 row blocks, so that the tiles at work share operands
struct TileWalk {
    int64_t mt, nt, all;
    __device__ __forceinline__ TileWalk(const GemmArgs& g, int width) {
        mt = (g.M + kTileM - 1) / kTileM;
        nt = (g.N + width - 1) / width;
        all = mt * nt * (g.twice ? 2 : 1);
    }
    __device__ __forceinline__ void at(int64_t t, int& prob, int64_t& m, int64_t& n) const {
        prob = t >= mt * nt;
        if (prob) t -= mt * nt;
        const int64_t group = t / (8 * nt), first = group * 8, rows = min((int64_t)8, mt - first);
        const int64_t in = t - group * 8 * nt;
        m = first + in % rows;
        n = in / rows;
    }
};

template <int BN, bool AT, bool BT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kTcThreads, 1)
    gemm_tc_kernel(const __grid_constant__ GemmArgs g, const __grid_constant__ TcMaps maps) {
    using S = TcTile<BN>;
    extern __shared__ unsigned char raw[];
    unsigned char* const ring = (unsigned char*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    TcBarriers& bar = *reinterpret_cast<TcBarriers*>(ring + S::kRing);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = cluster_rank();
    const bool gated = g.e.kind == FINISH_GATED;
    const int width = gated ? BN / 2 : BN;
    const TileWalk walk(g, width);
    const int64_t first = blockIdx.x / 2, step = gridDim.x / 2;
    const int slices = (g.K + kSliceK - 1) / kSliceK, all = slices * g.segs;

    if (warp == 0 && lane == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            mbar_init(&bar.full[i], 1);
            mbar_init(&bar.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bar.done[i], 1);
            mbar_init(&bar.free[i], 8);  // the finishing warps of both CTAs
        }
        mbar_init(&bar.drain, 1);
        mbar_fence_init();
    }
    if (warp == 2) tc2_alloc(&bar.tmem, S::kTmem);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = bar.tmem;

    if (warp == 0) {  // ---- copies
        if (one_lane()) {
            int64_t n = 0;  // slices so far
            bool ok = true;
            for (int64_t t = first; t < walk.all && ok; t += step) {
                int prob;
                int64_t mt, nt;
                walk.at(t, prob, mt, nt);
                const int m0 = (int)(mt * kTileM + rank * 128);
                const int n0 = (int)(nt * width) + (gated ? 0 : (int)rank * (BN / 2));
                for (int c = 0; c < all; ++c, ++n) {
                    const int slot = (int)(n % S::kStages);
                    const uint32_t use = (uint32_t)(n / S::kStages);
                    if (use > 0 && !(ok = mbar_wait(&bar.empty[slot], (use - 1) & 1, g.status))) break;
                    const int seg = c >= slices, k = (c - seg * slices) * kSliceK;
                    unsigned char* const a = ring + slot * (S::kA + S::kB);
                    unsigned char* const b = a + S::kA;
                    if (rank == 0) mbar_arrive_expect_tx(&bar.full[slot], 2 * (S::kA + S::kB));
                    const uint32_t full = peer_u32(&bar.full[slot], 0);
                    const CUtensorMap* const am = &maps.a[seg + prob];
                    const CUtensorMap* const bm = &maps.b[gated ? (int)rank : seg];
                    if (AT) {
                        for (int i = 0; i < 2; ++i) tma_box_pair(a + i * 8192, am, m0 + 64 * i, k, full);
                    } else {
                        tma_box_pair(a, am, k, m0, full);
                    }
                    if (BT) {
                        for (int i = 0; i < BN / 128; ++i) tma_box_pair(b + i * 8192, bm, n0 + 64 * i, k, full);
                    } else {
                        tma_box_pair(b, bm, k, n0, full);
                    }
                }
            }
            if (!ok && rank == 0) {  // (what is in flight lands before the CTA ends)
                for (int64_t i = n > S::kStages ? n - S::kStages : 0; i < n; ++i)
                    mbar_wait(&bar.full[i % S::kStages], (uint32_t)(i / S::kStages) & 1, g.status, 50000000LL);
            }
        }
        __syncwarp();
    } else if (warp == 1 && rank == 0) {  // ---- products
        const uint32_t id = idesc_bf16_f32(256, BN) | (AT ? 1u << 15 : 0) | (BT ? 1u << 16 : 0);
        if (one_lane()) {
            int64_t n = 0;
            uint32_t i = 0;  // tiles so far
            bool ok = true;
            for (int64_t t = first; t < walk.all && ok; t += step, ++i) {
                const uint32_t buf = i & 1, use = i >> 1, d = tmem + buf * BN;
                if (use > 0 && !(ok = mbar_wait(&bar.free[buf], (use - 1) & 1, g.status))) break;
                tc_fence_after();
                for (int c = 0; c < all; ++c, ++n) {
                    const int slot = (int)(n % S::kStages);
                    if (!(ok = mbar_wait(&bar.full[slot], (uint32_t)(n / S::kStages) & 1, g.status))) break;
                    tc_fence_after();
                    const uint32_t at = smem_u32(ring + slot * (S::kA + S::kB));
                    const uint64_t ad = operand_desc(at, AT), bd = operand_desc(at + S::kA, BT);
#pragma unroll
                    for (int k = 0; k < kSliceK / 16; ++k)
                        tc2_mma(d, ad + k * (AT ? 128 : 2), bd + k * (BT ? 128 : 2), id, c > 0 || k > 0);
                    tc2_commit(&bar.empty[slot]);
                }
                tc2_commit(&bar.done[buf]);
            }
            if (!ok) {
                tc2_commit(&bar.drain);
                mbar_wait(&bar.drain, 0, g.status, 50000000LL);
            }
        }
        __syncwarp();
    } else if (warp >= 2) {  // ---- results
        const int quarter = warp & 3;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        uint32_t i = 0;
        for (int64_t t = first; t < walk.all; t += step, ++i) {
            int prob;
            int64_t mt, nt;
            walk.at(t, prob, mt, nt);
            const uint32_t buf = i & 1, use = i >> 1, d = tmem + buf * BN + lanes;
            bool ok = true;
            if (lane == 0) ok = mbar_wait(&bar.done[buf], use & 1, g.status);
            if (!__shfl_sync(0xffffffffu, ok, 0)) break;
            tc_fence_after();
            const int64_t m = mt * kTileM + rank * 128 + quarter * 32 + lane;
            const int n0 = (int)(nt * width);
            Finish e = g.e;
            if (prob) {
                e.out = e.out2;
                e.out_row = e.out2_row;
            }
            for (int c = 0; c < width && n0 + c < g.N; c += 32) {
                float z[32];
                tc_ld32(d + c, z);
                if (gated) {
                    float u[32];
                    tc_ld32(d + BN / 2 + c, u);
                    if (m < g.M) epilogue_gated<bf16_t, 32>(e, m, n0 + c, g.N, z, u);
                } else if (m < g.M) {
                    epilogue_one<bf16_t, 32>(e, m, n0 + c, g.N, z);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_peer(peer_u32(&bar.free[buf], 0));
        }
    }
    __syncthreads();
    cluster_sync_all();
    if (warp == 2) tc2_dealloc(tmem, S::kTmem);
}

// A matrix [rows, cols] of bfloat16 in boxes of 64 columns
bool make_map(CUtensorMap* map, const fe_mat& m, int64_t rows, int64_t cols, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(rows > 1 ? m.row : (cols + 7) / 8 * 8) * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, step[2] = {1, 1};
    const EncodeTiled encode = encode_tiled();
    return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, m.p, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN, bool AT, bool BT>
cudaError_t launch_pairs(const GemmArgs& g, int num_sms, cudaStream_t st) {
    using S = TcTile<BN>;
    TcMaps maps{};
    const bool gated = g.e.kind == FINISH_GATED;
    for (int i = 0; i < 2; ++i) {
        if (i == 0 || g.segs == 2 || g.twice) {
            if (!(AT ? make_map(&maps.a[i], g.a[i], g.K, g.M, 64) : make_map(&maps.a[i], g.a[i], g.M, g.K, 128))) return cudaErrorInvalidValue;
        }
        if (i == 0 || g.segs == 2 || gated) {
            if (!(BT ? make_map(&maps.b[i], g.b[i], g.K, g.N, 64) : make_map(&maps.b[i], g.b[i], g.N, g.K, BN / 2))) return cudaErrorInvalidValue;
        }
    }
    const int width = gated ? BN / 2 : BN;
    const int64_t tiles = (g.M + kTileM - 1) / kTileM * ((g.N + width - 1) / width) * (g.twice ? 2 : 1);
    const int64_t pairs = tiles < num_sms / 2 ? tiles : num_sms / 2;
    return launch_k(gemm_tc_kernel<BN, AT, BT>, dim3((unsigned)(2 * pairs)), dim3(kTcThreads), S::kSmem, st, false, g, maps);
}

template <bool AT, bool BT>
cudaError_t launch_tiles(const GemmArgs& g, int num_sms, cudaStream_t st) {
    const int64_t mt = (g.M + kTileM - 1) / kTileM * (g.twice ? 2 : 1), pairs = num_sms / 2;
    const int w = g.e.kind == FINISH_GATED ? 2 : 1;
    const auto rounds = [&](int bn) { return (mt * ((g.N + bn / w - 1) / (bn / w)) + pairs - 1) / pairs; };
    // narrow tiles where they take less than the wide ones' rounds: a narrow tile costs some 0.6 of a wide one
    if (rounds(128) * 6 < rounds(256) * 10) return launch_pairs<128, AT, BT>(g, num_sms, st);
    return launch_pairs<256, AT, BT>(g, num_sms, st);
}

// Rows that TMA cannot read (off 16-byte boundaries, repeated) as rows that it can
__global__ void __launch_bounds__(256) pack_rows_kernel(const bf16_t* src, int64_t src_row, bf16_t* dst, int64_t dst_row, int64_t rows, int64_t cols) {
    const int64_t strips = (cols + 255) / 256, all = rows * strips;
    for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
        const int64_t r = u / strips, c = u % strips * 256 + threadIdx.x;
        if (c < cols) dst[r * dst_row + c] = src[r * src_row + c];
    }
}

template <int BN, bool AT, bool BT>
cudaError_t allow() {
    return cudaFuncSetAttribute(gemm_tc_kernel<BN, AT, BT>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcTile<BN>::kSmem);
}

}  // namespace

cudaError_t gemm_tc_prepare() {
    cudaError_t e;
    if ((e = allow<256, false, false>()) != cudaSuccess || (e = allow<256, false, true>()) != cudaSuccess) return e;
    if ((e = allow<256, true, true>()) != cudaSuccess || (e = allow<128, false, false>()) != cudaSuccess) return e;
    if ((e = allow<128, false, true>()) != cudaSuccess) return e;
    return allow<128, true, true>();
}

bool gemm_tc_reads(const fe_mat& m, int64_t rows, int64_t cols) {
    return ((uintptr_t)m.p & 15) == 0 && (rows <= 1 || (m.row % 8 == 0 && m.row >= cols && m.row < (int64_t)1 << 38));
}

cudaError_t launch_pack_rows(const fe_mat& src, const fe_mat& dst, int64_t rows, int64_t cols, int num_sms, cudaStream_t st) {
    const int64_t units = rows * ((cols + 255) / 256), most = (int64_t)num_sms * 32;
    return launch_k(pack_rows_kernel, dim3((unsigned)(units < most ? units : most)), dim3(256), 0, st, false, (const bf16_t*)src.p, src.row,
                    (bf16_t*)dst.p, dst.row, rows, cols);
}

cudaError_t launch_gemm_tc(const GemmArgs& g, int num_sms, cudaStream_t st) {
    if (g.a_t) return launch_tiles<true, true>(g, num_sms, st);
    return g.b_t ? launch_tiles<false, true>(g, num_sms, st) : launch_tiles<false, false>(g, num_sms, st);
}

}  // namespace fe
