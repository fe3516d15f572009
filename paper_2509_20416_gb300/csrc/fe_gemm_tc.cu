// Matrix products of bfloat16 on the tensor cores (fe_layer.h's products and their gradients): C = A B^T
// with either operand stored by rows or by its summed index, float32 sums in tensor memory.
//
// Persistent pairs of CTAs (cta_group::2) make tiles of 256 x BN, BN 128 to 256: each CTA brings, by TMA, 128
// rows of A and BN / 2 of B in slices of 64 of the summed index, so that an SM reads half of what a CTA of
// its own would for the same products. Warp 0 copies, warp 1 of the first CTA issues the products, warps 2
// to 9 finish a tile (bias, activation, residual, gate, rounding) while the next one is summed in the
// other half of tensor memory. The MN-major operand forms spare the gradients every transpose:
// dx = dz w reads w by columns, dw = dz^T x both operands.
//
// Measured (GB300): 4093 x 5120 x 5120 119 to 124 us (1730 to 1810 TFLOP/s; cuBLAS 119 to 126 on the same boxes),
// with gelu, bias, residual and the float32 pre-activation 136; a gated pair of 14336 x 4096 from 4093 rows 482 us
// (1990 TFLOP/s), 523 with both products stored; the gradients' products 1650 to 1910 TFLOP/s. Long steps are bound by
// the card's power (1550 TFLOP/s over a block's forward and backward pass). Five slices in flight instead of six cost 4 %.
//
// BN is the width whose rounds of tiles over the pairs are shortest (fe_gemm_plan.h): 16 x 16 tiles of 256 take 76 pairs 4
// rounds where 3.4 would hold them, 16 x 19 of 224 take 4 rounds of 7/8.
#include "fe_gemm_plan.h"
#include "fe_gemm_tc.cuh"
#include "fe_tensor_map.h"

namespace fe {

namespace {

constexpr int kTcThreads = 64 + 32 * kFinishWarps;

// How long a finishing warp waits for a tile, besides what any wait gets: a weight's gradient sums up to 2^24 slices
// in one tile, at 230 ns each where a pair works alone, 750 where the copies of all pairs come from memory.
constexpr int64_t kSliceBudgetNs = 2000;

constexpr int kStaging = kFinishWarps * 4096;  // a warp's 32 x 32 floats
constexpr int kTcSmem = kTcRing + kStaging + 1024 /* alignment */ + 512;
static_assert(kTcSmem <= 227 * 1024, "shared memory of a CTA");

struct TcBarriers {
    uint64_t full[kTcStages], empty[kTcStages], done[2], free[2], drain;
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

// four consecutive columns of bfloat16 as they are stored, and of float32
__device__ __forceinline__ uint2 load4(const bf16_t* p, int have, bool vec) {
    if (vec && have >= 4) return *reinterpret_cast<const uint2*>(p);
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i < have ? p[i].bits : 0u;
    return make_uint2(x[0] | x[1] << 16, x[2] | x[3] << 16);
}
__device__ __forceinline__ float4 load4(const float* p, int have, bool vec) {
    if (vec && have >= 4) return *reinterpret_cast<const float4*>(p);
    return make_float4(have > 0 ? p[0] : 0.f, have > 1 ? p[1] : 0.f, have > 2 ? p[2] : 0.f, have > 3 ? p[3] : 0.f);
}
__device__ __forceinline__ void widen4(const uint2& x, float* f) {
    f[0] = __uint_as_float(x.x << 16), f[1] = __uint_as_float(x.x & 0xFFFF0000u);
    f[2] = __uint_as_float(x.y << 16), f[3] = __uint_as_float(x.y & 0xFFFF0000u);
}
__device__ __forceinline__ void store4(bf16_t* p, int have, bool vec, const float* f) {
    if (vec && have >= 4) {
        *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) store_one(p + i, f[i]);
    }
}
__device__ __forceinline__ void store4(float* p, int have, bool vec, const float* f) {
    if (vec && have >= 4) {
        *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) p[i] = f[i];
    }
}

// A warp's 32 x 32 block turned from a row a lane (as tensor memory gives it) to four columns a lane, 8
// lanes a row, so that rows meet global memory in whole sectors. 16-byte chunk c of row r lies at c ^ (r & 7).
// What comes before it branches by lane at ragged edges; the load from tensor memory is the warp's as one.
__device__ __forceinline__ void stage_rows(float* buf, uint32_t d, int lane) {
    float z[32];
    __syncwarp();
    tc_ld32(d, z);
#pragma unroll
    for (int c = 0; c < 8; ++c)
        *reinterpret_cast<float4*>(buf + lane * 32 + ((c ^ (lane & 7)) << 2)) = make_float4(z[4 * c], z[4 * c + 1], z[4 * c + 2], z[4 * c + 3]);
    __syncwarp();
}
__device__ __forceinline__ void staged(const float* buf, int row, int chunk, float* f) {
    const float4 x = *reinterpret_cast<const float4*>(buf + row * 32 + ((chunk ^ (row & 7)) << 2));
    f[0] = x.x, f[1] = x.y, f[2] = x.z, f[3] = x.w;
}

// A warp's part of a tile: 32 rows from m0 on, of which it takes columns n0 + 32 half, + 64, ... below n0 +
// width. A lane has four columns of every fourth row; the rows are `left` (none: 0).
struct WarpTile {
    const Finish& e;
    uint32_t d, d2;  // tensor memory: the product, and the gated pair's second
    int64_t m0;
    int left, n0, end, lane;  // end: the first column behind the tile
    float* buf;
    __device__ __forceinline__ int row(int i) const { return 4 * i + (lane >> 3); }
    __device__ __forceinline__ int chunk() const { return lane & 7; }
    __device__ __forceinline__ bool inside(int c) const { return n0 + c < end; }
    __device__ __forceinline__ int have(int c) const { return end - n0 - c - 4 * chunk(); }
    template <typename T>
    __device__ __forceinline__ T* at(void* base, int64_t stride, int c) const {
        return (T*)base + (m0 + row(0)) * stride + n0 + c + 4 * chunk();
    }
};

// act(z + bias) + res. What the next block reads of the residual is in flight while a block is finished.
__device__ __forceinline__ void residual_rows(const WarpTile& w, int c, uint2* r) {
    const bf16_t* p = w.at<bf16_t>((void*)w.e.res, w.e.res_row, c);
    const int have = w.inside(c) ? w.have(c) : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = load4(p + 4 * i * w.e.res_row, w.row(i) < w.left ? have : 0, w.e.vec);
}
template <typename Wait>
__device__ __forceinline__ bool finish_plain(const WarpTile& w, int half, const Wait& wait) {
    const Finish& e = w.e;
    uint2 next[8], r[8];
    if (e.res) residual_rows(w, half * 32, next);
    if (!wait()) return false;
    for (int c = half * 32; w.inside(c); c += 64) {
        const int have = w.have(c);
        float b[4] = {0.f, 0.f, 0.f, 0.f};
        if (e.bias) widen4(load4((const bf16_t*)e.bias + w.n0 + c + 4 * w.chunk(), have, e.vec), b);
        if (e.res) {
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = next[i];
            residual_rows(w, c + 64, next);
        }
        stage_rows(w.buf, w.d + c, w.lane);
        float* pre = w.at<float>(e.pre, e.pre_row, c);
        bf16_t* out = w.at<bf16_t>(e.out, e.out_row, c);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float z[4];
            staged(w.buf, w.row(i), w.chunk(), z);
            if (w.row(i) >= w.left) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) z[j] += b[j];
            if (e.pre) store4(pre + 4 * i * e.pre_row, have, e.vec, z);
            if (e.act != FE_ACT_NONE) {
#pragma unroll
                for (int j = 0; j < 4; ++j) z[j] = act_value<true>(e.act, z[j]);
            }
            if (e.res) {
                float t[4];
                widen4(r[i], t);
#pragma unroll
                for (int j = 0; j < 4; ++j) z[j] += t[j];
            }
            store4(out + 4 * i * e.out_row, have, e.vec, z);
        }
        __syncwarp();  // (the buffer's next block)
    }
    return true;
}

// act(z) u
__device__ __forceinline__ void finish_gated(const WarpTile& w, int half) {
    const Finish& e = w.e;
    for (int c = half * 32; w.inside(c); c += 64) {
        const int have = w.have(c);
        float u[8][4];
        stage_rows(w.buf, w.d2 + c, w.lane);
#pragma unroll
        for (int i = 0; i < 8; ++i) staged(w.buf, w.row(i), w.chunk(), u[i]);
        __syncwarp();
        stage_rows(w.buf, w.d + c, w.lane);
        float *pre = w.at<float>(e.pre, e.pre_row, c), *pre2 = w.at<float>(e.pre2, e.pre2_row, c);
        bf16_t* out = w.at<bf16_t>(e.out, e.out_row, c);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float g[4];
            staged(w.buf, w.row(i), w.chunk(), g);
            if (w.row(i) >= w.left) continue;
            if (e.pre) {
                store4(pre + 4 * i * e.pre_row, have, e.vec, g);
                store4(pre2 + 4 * i * e.pre2_row, have, e.vec, u[i]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) g[j] = act_value<true>(e.act, g[j]) * u[i][j];
            store4(out + 4 * i * e.out_row, have, e.vec, g);
        }
        __syncwarp();
    }
}

// The gradients of a gated pair. A lane's stored products of a row of the next block are copied (cp.async) into the
// place of the row that it has just read, which it alone writes and reads: 8 KB a warp, 64 KB an SM in flight.
__device__ __forceinline__ void pair_row(const WarpTile& w, int c, int i, float4* slot) {
    const int have = w.inside(c) && w.row(i) < w.left ? w.have(c) : 0;
    if (have > 0) {
        const float* g = w.at<float>(w.e.pre, w.e.pre_row, c) + 4 * i * w.e.pre_row;
        const float* u = w.at<float>(w.e.pre2, w.e.pre2_row, c) + 4 * i * w.e.pre2_row;
        if (w.e.vec && have >= 4) {
            cp_async16(smem_u32(slot + 64 * i), g, true);
            cp_async16(smem_u32(slot + 64 * i + 32), u, true);
        } else {
            slot[64 * i] = load4(g, have, false);
            slot[64 * i + 32] = load4(u, have, false);
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
}
template <typename Wait>
__device__ __forceinline__ bool finish_gated_grad(const WarpTile& w, int half, const Wait& wait, float4* slots) {
    const Finish& e = w.e;
    float4* const slot = slots + w.lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) pair_row(w, half * 32, i, slot);
    const bool ok = wait();
    for (int c = half * 32; ok && w.inside(c); c += 64) {
        const int have = w.have(c);
        stage_rows(w.buf, w.d + c, w.lane);
        bf16_t *out = w.at<bf16_t>(e.out, e.out_row, c), *out2 = w.at<bf16_t>(e.out2, e.out2_row, c),
               *out3 = w.at<bf16_t>(e.out3, e.out3_row, c);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float z[4];
            asm volatile("cp.async.wait_group 7;" ::: "memory");
            const float4 cg = slot[64 * i], cu = slot[64 * i + 32];
            float g[4] = {cg.x, cg.y, cg.z, cg.w}, u[4] = {cu.x, cu.y, cu.z, cu.w};
            pair_row(w, c + 64, i, slot);
            staged(w.buf, w.row(i), w.chunk(), z);
            if (w.row(i) >= w.left || have <= 0) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float v, dv;
                act_both<true>(e.act, g[j], v, dv);
                g[j] = z[j] * v;
                z[j] *= u[j] * dv;
                u[j] *= v;
            }
            store4(out + 4 * i * e.out_row, have, e.vec, z);
            store4(out2 + 4 * i * e.out2_row, have, e.vec, g);
            store4(out3 + 4 * i * e.out3_row, have, e.vec, u);
        }
        __syncwarp();
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    return ok;
}

template <bool AT, bool BT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kTcThreads, 1)
    gemm_tc_kernel(const __grid_constant__ GemmArgs g, const __grid_constant__ TcMaps maps, const TcWidth shape) {
    const int BN = shape.bn, stages = shape.stages, stage_bytes = kSliceA + shape.b_bytes;
    extern __shared__ unsigned char raw[];
    unsigned char* const ring = (unsigned char*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    TcBarriers& bar = *reinterpret_cast<TcBarriers*>(ring + kTcRing + kStaging);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = cluster_rank();
    const bool gated = g.e.kind == FINISH_GATED;
    const int width = gated ? BN / 2 : BN;
    const TileWalk walk(g, width);
    const int64_t first = blockIdx.x / 2, step = gridDim.x / 2;
    const int slices = (g.K + kSliceK - 1) / kSliceK, all = slices * g.segs;

    if (warp == 0 && lane == 0) {
        for (int i = 0; i < stages; ++i) {
            mbar_init(&bar.full[i], 1);
            mbar_init(&bar.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bar.done[i], 1);
            mbar_init(&bar.free[i], 2 * kFinishWarps);  // the finishing warps of both CTAs
        }
        mbar_init(&bar.drain, 1);
        mbar_fence_init();
    }
    if (warp == 2) tc2_alloc(&bar.tmem, 512);  // two accumulators of up to 256 columns
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = bar.tmem;

    if (warp == 0) {  // ---- copies
        if (one_lane()) {
            int64_t n = 0;  // slices so far
            int slot = 0;
            uint32_t phase = 0;  // of the slot's current use
            bool ok = true;
            for (int64_t t = first; t < walk.all && ok; t += step) {
                int prob;
                int64_t mt, nt;
                walk.at(t, prob, mt, nt);
                const int m0 = (int)(mt * kTileM + rank * 128);
                const int n0 = (int)(nt * width) + (gated ? 0 : (int)rank * (BN / 2));
                for (int c = 0; c < all; ++c, ++n) {
                    if (n >= stages && !(ok = mbar_wait(&bar.empty[slot], phase ^ 1, g.status))) break;
                    const int seg = c >= slices, k = (c - seg * slices) * kSliceK;
                    unsigned char* const a = ring + slot * stage_bytes;
                    unsigned char* const b = a + kSliceA;
                    if (rank == 0) mbar_arrive_expect_tx(&bar.full[slot], 2 * stage_bytes);
                    const uint32_t full = peer_u32(&bar.full[slot], 0);
                    const CUtensorMap* const am = &maps.a[seg + prob];
                    const CUtensorMap* const bm = &maps.b[gated ? (int)rank : seg];
                    if (AT) {
                        for (int i = 0; i < 2; ++i) tma_box_pair(a + i * 8192, am, m0 + 64 * i, k, full);
                    } else {
                        tma_box_pair(a, am, k, m0, full);
                    }
                    if (BT) {  // (whole groups of 64 columns: of the last one the product reads what it needs)
                        for (int i = 0; i < shape.b_bytes / 8192; ++i) tma_box_pair(b + i * 8192, bm, n0 + 64 * i, k, full);
                    } else {
                        tma_box_pair(b, bm, k, n0, full);
                    }
                    if (++slot == stages) slot = 0, phase ^= 1;
                }
            }
            if (!ok && rank == 0) {  // (what is in flight lands before the CTA ends)
                for (int64_t i = n > stages ? n - stages : 0; i < n; ++i)
                    mbar_wait(&bar.full[i % stages], (uint32_t)(i / stages) & 1, g.status, 50000000LL);
            }
        }
        __syncwarp();
    } else if (warp == 1 && rank == 0) {  // ---- products
        const uint32_t id = idesc_bf16_f32(256, BN) | (AT ? 1u << 15 : 0) | (BT ? 1u << 16 : 0);
        if (one_lane()) {
            uint32_t i = 0;  // tiles so far
            int slot = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int64_t t = first; t < walk.all && ok; t += step, ++i) {
                const uint32_t buf = i & 1, use = i >> 1, d = tmem + buf * 256;
                if (use > 0 && !(ok = mbar_wait(&bar.free[buf], (use - 1) & 1, g.status))) break;
                tc_fence_after();
                for (int c = 0; c < all; ++c) {
                    if (!(ok = mbar_wait(&bar.full[slot], phase, g.status))) break;
                    tc_fence_after();
                    const uint32_t at = smem_u32(ring + slot * stage_bytes);
                    const uint64_t ad = operand_desc(at, AT), bd = operand_desc(at + kSliceA, BT);
#pragma unroll
                    for (int k = 0; k < kSliceK / 16; ++k)
                        tc2_mma(d, ad + k * (AT ? 128 : 2), bd + k * (BT ? 128 : 2), id, c > 0 || k > 0);
                    tc2_commit(&bar.empty[slot]);
                    if (++slot == stages) slot = 0, phase ^= 1;
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
        const int quarter = warp & 3, half = (warp - 2) >> 2;  // a quarter of the rows, every second 32 columns
        float* const buf_rows = (float*)(ring + kTcRing) + (warp - 2) * 1024;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        Finish e = g.e;
        uint32_t i = 0;
        for (int64_t t = first; t < walk.all; t += step, ++i) {
            int prob;
            int64_t mt, nt;
            walk.at(t, prob, mt, nt);
            const uint32_t buf = i & 1, use = i >> 1, d = tmem + buf * 256 + lanes;
            const auto wait = [&] {
                bool ok = true;
                if (lane == 0) ok = mbar_wait(&bar.done[buf], use & 1, g.status, kWaitBudgetNs + all * kSliceBudgetNs);
                ok = __shfl_sync(0xffffffffu, ok, 0);
                tc_fence_after();
                return ok;
            };
            if (prob) {
                e.out = g.e.out2;
                e.out_row = g.e.out2_row;
            }
            const int64_t m0 = mt * kTileM + rank * 128 + quarter * 32;
            const WarpTile w{e, d, d + BN / 2, m0, (int)(m0 < g.M ? min((int64_t)32, g.M - m0) : 0), (int)(nt * width), (int)min((int64_t)g.N, (nt + 1) * width), lane, buf_rows};
            if (gated) {
                if (!wait()) break;
                finish_gated(w, half);
            } else if (e.kind == FINISH_GATED_GRAD) {
                if (!finish_gated_grad(w, half, wait, (float4*)(ring + kTcRing - kPairs) + (warp - 2) * 512)) break;
            } else if (!finish_plain(w, half, wait)) {
                break;
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_peer(peer_u32(&bar.free[buf], 0));
        }
    }
    __syncthreads();
    cluster_sync_all();
    if (warp == 2) tc2_dealloc(tmem, 512);
}

template <bool AT, bool BT>
cudaError_t launch_tiles(const GemmArgs& g, int num_sms, cudaStream_t st) {
    const bool gated = g.e.kind == FINISH_GATED;
    const TcWidth shape = tc_width(g.M, g.N, gated, g.twice, g.e.kind == FINISH_GATED_GRAD, BT, num_sms);
    const int bn = shape.bn;
    TcMaps maps{};
    for (int i = 0; i < 2; ++i) {
        if (i == 0 || g.segs == 2 || g.twice) {
            if (!(AT ? tensor_map_bf16(&maps.a[i], g.a[i], g.K, g.M, 64) : tensor_map_bf16(&maps.a[i], g.a[i], g.M, g.K, 128))) return cudaErrorInvalidValue;
        }
        if (i == 0 || g.segs == 2 || gated) {
            if (!(BT ? tensor_map_bf16(&maps.b[i], g.b[i], g.K, g.N, 64) : tensor_map_bf16(&maps.b[i], g.b[i], g.N, g.K, bn / 2))) return cudaErrorInvalidValue;
        }
    }
    const int64_t tiles = tc_tiles(g.M, g.N, gated, g.twice, bn), pairs = num_sms / 2, n = tiles < pairs ? tiles : pairs;
    return launch_k(gemm_tc_kernel<AT, BT>, dim3((unsigned)(2 * n)), dim3(kTcThreads), kTcSmem, st, false, g, maps, shape);
}

// Rows that TMA cannot read (off 16-byte boundaries, repeated) as rows that it can
__global__ void __launch_bounds__(256) pack_rows_kernel(const bf16_t* src, int64_t src_row, bf16_t* dst, int64_t dst_row, int64_t rows, int64_t cols) {
    const int64_t strips = (cols + 255) / 256, all = rows * strips;
    for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
        const int64_t r = u / strips, c = u % strips * 256 + threadIdx.x;
        if (c < cols) dst[r * dst_row + c] = src[r * src_row + c];
    }
}

template <bool AT, bool BT>
cudaError_t allow() {
    return cudaFuncSetAttribute(gemm_tc_kernel<AT, BT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kTcSmem);
}

}  // namespace

cudaError_t gemm_tc_prepare() {
    cudaError_t e;
    if ((e = allow<false, false>()) != cudaSuccess || (e = allow<false, true>()) != cudaSuccess) return e;
    return allow<true, true>();
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
