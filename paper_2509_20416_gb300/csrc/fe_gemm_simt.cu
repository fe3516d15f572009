// Matrix products on the CUDA cores: float32 throughout, any size, stride and alignment, either
// operand with its summed index as columns or as rows (fe_layer.h's products and their gradients).
//
// A CTA of 256 threads makes a BM x BN tile, a thread BM/16 x BN/16 of it in registers: per step of
// the summed index it reads (BM + BN) / 16 floats from shared memory for BM BN / 256 products. The
// products go in pairs of columns (fma.rn.f32x2). Slices of 16 steps alternate between two buffers;
// the next slice's loads (the next two's of a small tile) are in flight while a slice is multiplied. Where
// there are few tiles a cluster divides the summed index, and its CTAs' sums are added in their order
// through distributed shared memory.
//
// Bound by issue and shared memory: 4096 cubed 2.5 ms (55 TFLOP/s, 70 % of the float32 units), 331 x 688 x 257 15 us
// (41 us without clusters). At most 8 rows: one row to 6144 of 4096 16 us (92 % of the copy rate).
#include "fe_gemm_plan.h"
#include "fe_gemm_tc.cuh"

namespace fe {

namespace {

constexpr int kBK = 16;

// One operand's slice of R rows (tile rows) x 16 steps. Stored by rows (summed index contiguous) a
// thread takes runs of 4 steps of a row, stored by steps (T) runs of 4 rows of a step.
template <int R, bool STEPS>
struct Slice {
    static constexpr int kRuns = R * kBK / 4 / 256;
    float v[kRuns][4];

    // Steps k0 on, of K, of the R rows from r0 on, of `rows` (STEPS: columns of the stored matrix); what lies
    // outside is 0. By rows, a tile of a gated pair (split > 0) takes its rows from `split` on from the second matrix.
    __device__ __forceinline__ void load(const fe_mat& m, int64_t r0, int64_t rows, int k0, int K, bool vec, int split,
                                         const fe_mat& second) {
#pragma unroll
        for (int i = 0; i < kRuns; ++i) {
            const int u = threadIdx.x + i * 256;
            if (!STEPS) {
                const int r = u / (kBK / 4), k = k0 + u % (kBK / 4) * 4;
                const bool two = split > 0 && r >= split;
                const int64_t row = r0 + (two ? r - split : r);
                const float* p = (const float*)(two ? second.p : m.p) + row * (two ? second.row : m.row) + k;
                run(p, row < rows ? K - k : 0, vec, v[i]);
            } else {
                const int k = u / (R / 4), r = u % (R / 4) * 4;
                const float* p = (const float*)m.p + (int64_t)(k0 + k) * m.row + r0 + r;
                const int64_t left = rows - r0 - r;
                run(p, k0 + k < K ? (left < 4 ? (int)left : 4) : 0, vec, v[i]);
            }
        }
    }
    __device__ __forceinline__ static void run(const float* p, int have, bool vec, float* f) {
        if (vec && have >= 4) {
            const float4 x = *reinterpret_cast<const float4*>(p);
            f[0] = x.x, f[1] = x.y, f[2] = x.z, f[3] = x.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = i < have ? p[i] : 0.f;
        }
    }
    __device__ __forceinline__ void store(float (*s)[R + 4]) const {
#pragma unroll
        for (int i = 0; i < kRuns; ++i) {
            const int u = threadIdx.x + i * 256;
            if (!STEPS) {
                const int r = u / (kBK / 4), k = u % (kBK / 4) * 4;
#pragma unroll
                for (int e = 0; e < 4; ++e) s[k + e][r] = v[i][e];
            } else {
                const int k = u / (R / 4), r = u % (R / 4) * 4;
                *reinterpret_cast<float4*>(&s[k][r]) = make_float4(v[i][0], v[i][1], v[i][2], v[i][3]);
            }
        }
    }
};

template <int N>
__device__ __forceinline__ void read_run(const float* s, float* f) {
    if constexpr (N == 4) {
        const float4 x = *reinterpret_cast<const float4*>(s);
        f[0] = x.x, f[1] = x.y, f[2] = x.z, f[3] = x.w;
    } else {
        const float2 x = *reinterpret_cast<const float2*>(s);
        f[0] = x.x, f[1] = x.y;
    }
}

template <int BM, int BN, bool AT, bool BT, int P>
__global__ void __launch_bounds__(256, BM == 128 ? 2 : 3)
    gemm_simt_kernel(const __grid_constant__ GemmArgs g, int a_vec, int b_vec, int ranks) {
    constexpr int HM = BM / 32, HN = BN / 32;  // a thread's rows and columns: HM and HN in each half of the tile
    constexpr bool SPLIT = BM == 64;  // tiles that a cluster may divide
    union Room {
        struct {
            float a[2][kBK][BM + 4], b[2][kBK][BN + 4];
        } slice;
        float part[SPLIT ? BM : 1][BN + 4];  // a cluster's CTA's sums
    };
    __shared__ Room room;
    auto& As = room.slice.a;
    auto& Bs = room.slice.b;
    const int width = g.e.kind == FINISH_GATED ? BN / 2 : BN;  // columns of the result in a tile
    const int64_t nt = (g.N + width - 1) / width, mt = (g.M + BM - 1) / BM;
    const int rank = ranks > 1 ? (int)cluster_rank() : 0;
    int64_t t = blockIdx.x / ranks;
    const int prob = t >= nt * mt;
    if (prob) t -= nt * mt;
    const int64_t m0 = t / nt * BM;
    const int n0 = (int)(t % nt) * width;
    // a warp's lanes are 4 x 8 threads of the tile, so that each of its reads of a slice is one turn of the banks
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int tx = warp % 2 * 8 + lane % 8, ty = warp / 2 * 4 + lane / 8;
    uint64_t acc[2 * HM][HN];
#pragma unroll
    for (int i = 0; i < 2 * HM; ++i)
#pragma unroll
        for (int j = 0; j < HN; ++j) acc[i][j] = 0;
    const int slices = (g.K + kBK - 1) / kBK, total = slices * g.segs;
    const int first = (int)((int64_t)total * rank / ranks), all = (int)((int64_t)total * (rank + 1) / ranks) - first;
    Slice<BM, AT> a[P];  // slices i + 1 to i + P, on their way while slice i is multiplied
    Slice<BN, BT> b[P];
    const auto fetch = [&](int s, int p) {
        if (s >= all) return;
        s += first;
        const int seg = s >= slices;
        const int k0 = (s - seg * slices) * kBK;
        a[p].load(g.a[seg + prob], m0, g.M, k0, g.K, a_vec, 0, g.a[0]);
        b[p].load(g.b[seg], n0, g.N, k0, g.K, b_vec, g.e.kind == FINISH_GATED ? width : 0, g.b[1]);
    };
#pragma unroll
    for (int p = 0; p < P; ++p) fetch(p, p);
    a[0].store(As[0]);
    b[0].store(Bs[0]);
    fetch(P, 0);
    __syncthreads();
    for (int s0 = 0; s0 < all; s0 += P) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int s = s0 + p;
            if (s >= all) break;
            const float(*sa)[BM + 4] = As[s & 1];
            const float(*sb)[BN + 4] = Bs[s & 1];
#pragma unroll
            for (int k = 0; k < kBK; ++k) {
                float av[2 * HM], bv[2 * HN];
                read_run<HM>(&sa[k][ty * HM], av);
                read_run<HM>(&sa[k][BM / 2 + ty * HM], av + HM);
                read_run<HN>(&sb[k][tx * HN], bv);
                read_run<HN>(&sb[k][BN / 2 + tx * HN], bv + HN);
#pragma unroll
                for (int i = 0; i < 2 * HM; ++i) {
                    const uint64_t ai = pair_f32(av[i]);
#pragma unroll
                    for (int j = 0; j < HN; ++j)
                        acc[i][j] = fma_x2(ai, pair_f32(__float_as_uint(bv[2 * j]), __float_as_uint(bv[2 * j + 1])), acc[i][j]);
                }
            }
            if (s + 1 < all) {
                const int q = (p + 1) % P;
                a[q].store(As[(s + 1) & 1]);
                b[q].store(Bs[(s + 1) & 1]);
                fetch(s + 1 + P, q);
                __syncthreads();
            }
        }
    }
    Finish e = g.e;
    if (prob) {
        e.out = e.out2;
        e.out_row = e.out2_row;
    }
    const auto finish = [&](int64_t m, float* z) {
        if (e.kind == FINISH_GATED) {
            epilogue_gated<HN>(e, m, n0 + tx * HN, g.N, z, z + HN);
        } else {
            epilogue_one<HN>(e, m, n0 + tx * HN, g.N, z);
            epilogue_one<HN>(e, m, n0 + BN / 2 + tx * HN, g.N, z + HN);
        }
    };
    const auto row_of = [&](int i) { return i < HM ? ty * HM + i : BM / 2 + ty * HM + i - HM; };
    if (SPLIT && ranks > 1) {  // the cluster's parts, added in their order; CTA ty mod ranks finishes a thread row's rows
        __syncthreads();       // (the slices have been read)
#pragma unroll
        for (int i = 0; i < 2 * HM; ++i) {
            float* const row = room.part[SPLIT ? row_of(i) : 0];
#pragma unroll
            for (int j = 0; j < HN; ++j) {
                const int c = 2 * j < HN ? tx * HN + 2 * j : BN / 2 + tx * HN + 2 * j - HN;
                row[c] = low_f32(acc[i][j]);
                row[c + 1] = high_f32(acc[i][j]);
            }
        }
        cluster_sync_all();
        for (int i = 0; i < 2 * HM && ty % ranks == rank; ++i) {
            float z[2 * HN] = {};
            for (int r = 0; r < ranks; ++r) {
                const uint32_t peer = peer_u32(room.part[SPLIT ? row_of(i) : 0], r);
#pragma unroll
                for (int j = 0; j < HN; ++j) {
                    z[j] += load_peer(peer + 4 * (tx * HN + j));
                    z[HN + j] += load_peer(peer + 4 * (BN / 2 + tx * HN + j));
                }
            }
            if (m0 + row_of(i) < g.M) finish(m0 + row_of(i), z);
        }
        cluster_sync_all();  // (the others have read this CTA's)
        return;
    }
#pragma unroll
    for (int i = 0; i < 2 * HM; ++i) {
        float z[2 * HN];
#pragma unroll
        for (int j = 0; j < HN; ++j) {
            z[2 * j] = low_f32(acc[i][j]);
            z[2 * j + 1] = high_f32(acc[i][j]);
        }
        if (m0 + row_of(i) < g.M) finish(m0 + row_of(i), z);
    }
}

// Products of at most 8 rows, bound by the weights' bytes: a CTA takes four rows of them (gated: two of either
// matrix), its eight warps an eighth of the summed index each; every load of the rows of A serves four rows.
constexpr int kDotRows = 4, kDotWarps = 8;
template <int MT, bool VEC>
__global__ void __launch_bounds__(kDotWarps * 32) dot_kernel(const __grid_constant__ GemmArgs g) {
    constexpr int V = VEC ? 4 : 1, U = MT <= 2 ? 4 : 2;  // elements of a load, loads of a row in flight
    __shared__ float sums[kDotWarps][MT][kDotRows];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const bool gated = g.e.kind == FINISH_GATED;
    const int64_t n0 = (int64_t)blockIdx.x * (gated ? 2 : 4);
    const float* w[kDotRows];
#pragma unroll
    for (int r = 0; r < kDotRows; ++r) {
        const int64_t n = min(n0 + (gated ? r % 2 : r), (int64_t)g.N - 1);
        const fe_mat& m = g.b[gated && r >= 2];
        w[r] = (const float*)m.p + n * m.row;
    }
    float acc[MT][kDotRows] = {};
    constexpr int turn = 32 * V * U;
    const auto load = [](const float* p, float* f) {
        if constexpr (VEC) {
            const float4 x = *reinterpret_cast<const float4*>(p);
            f[0] = x.x, f[1] = x.y, f[2] = x.z, f[3] = x.w;
        } else {
            f[0] = *p;
        }
    };
    for (int64_t k0 = (int64_t)warp * turn; k0 < g.K; k0 += kDotWarps * turn) {
        float x[kDotRows][U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t k = k0 + (u * 32 + lane) * V;
#pragma unroll
            for (int r = 0; r < kDotRows; ++r) {
#pragma unroll
                for (int i = 0; i < V; ++i) x[r][u][i] = 0.f;
                if (k < g.K) load(w[r] + k, x[r][u]);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t k = k0 + (u * 32 + lane) * V;
            if (k >= g.K) continue;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if (m >= g.M) break;
                float a[V];
                load((const float*)g.a[0].p + m * g.a[0].row + k, a);
#pragma unroll
                for (int r = 0; r < kDotRows; ++r)
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[m][r] = fmaf(a[i], x[r][u][i], acc[m][r]);
            }
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < kDotRows; ++r) {
            const float s = warp_sum(acc[m][r]);
            if (lane == 0) sums[warp][m][r] = s;
        }
    __syncthreads();
    const int r = threadIdx.x % kDotRows, m = threadIdx.x / kDotRows;
    if (m >= MT || m >= g.M) return;
    const auto total = [&](int row) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < kDotWarps; ++i) s += sums[i][m][row];
        return s;
    };
    if (gated) {
        float z = total(r % 2), u = total(2 + r % 2);
        if (r < 2) epilogue_gated<1>(g.e, m, (int)n0 + r, g.N, &z, &u);
    } else {
        float z = total(r);
        epilogue_plain<1>(g.e, m, (int)n0 + r, g.N, &z);
    }
}

// runs of 4 elements on their own boundary
bool runs_of_4(const fe_mat& m) { return ((uintptr_t)m.p & 15) == 0 && m.row % 4 == 0; }

template <int MT>
cudaError_t launch_dot(const GemmArgs& g, cudaStream_t st) {
    const int per = g.e.kind == FINISH_GATED ? 2 : 4;
    const bool vec = g.K % 4 == 0 && runs_of_4(g.a[0]) && runs_of_4(g.b[0]) && (per == 4 || runs_of_4(g.b[1]));
    return launch_k(vec ? dot_kernel<MT, true> : dot_kernel<MT, false>, dim3((unsigned)((g.N + per - 1) / per)), dim3(kDotWarps * 32), 0, st, false, g);
}

template <int BM, int BN, bool AT, bool BT>
cudaError_t launch_tile(const GemmArgs& g, int num_sms, cudaStream_t st) {
    const int width = g.e.kind == FINISH_GATED ? BN / 2 : BN;
    const int64_t tiles = ((g.M + BM - 1) / BM) * ((g.N + width - 1) / width) * (g.twice ? 2 : 1);
    // CTAs of a tile: as many as two an SM hold, with eight slices each at least
    const int64_t slices = ((int64_t)g.K + kBK - 1) / kBK * g.segs;
    int ranks = 1;
    while (BM == 64 && ranks < 8 && tiles * ranks <= num_sms && slices >= ranks * 2 * 8) ranks *= 2;
    if (tiles > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    const int na = g.segs == 2 || g.twice ? 2 : 1, nb = g.segs == 2 || g.e.kind == FINISH_GATED ? 2 : 1;
    bool av = true, bv = true;
    for (int i = 0; i < na; ++i) av = av && runs_of_4(g.a[i]);
    for (int i = 0; i < nb; ++i) bv = bv && runs_of_4(g.b[i]);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * ranks));
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ranks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ranks > 1;
    return cudaLaunchKernelEx(&cfg, gemm_simt_kernel<BM, BN, AT, BT, BM == 64 ? 2 : 1>, g, (int)av, (int)bv, ranks);
}

template <bool AT, bool BT>
cudaError_t launch_layout(const GemmArgs& g, int num_sms, cudaStream_t st) {
    if (simt_large(g.M, g.N, g.e.kind == FINISH_GATED, g.twice, num_sms)) return launch_tile<128, 128, AT, BT>(g, num_sms, st);
    return launch_tile<64, 64, AT, BT>(g, num_sms, st);
}

}  // namespace

cudaError_t launch_gemm_simt(const GemmArgs& g, int num_sms, cudaStream_t st) {
    if (!g.a_t && !g.b_t && g.segs == 1 && g.M <= 8 && g.e.kind != FINISH_GATED_GRAD)
        return g.M == 1 ? launch_dot<1>(g, st) : g.M == 2 ? launch_dot<2>(g, st) : g.M <= 4 ? launch_dot<4>(g, st) : launch_dot<8>(g, st);
    if (g.a_t) return launch_layout<true, true>(g, num_sms, st);  // (a weight's gradient: both by steps)
    return g.b_t ? launch_layout<false, true>(g, num_sms, st) : launch_layout<false, false>(g, num_sms, st);
}

}  // namespace fe
