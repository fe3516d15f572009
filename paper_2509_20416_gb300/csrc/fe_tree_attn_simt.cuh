// Attention over the cache on the CUDA cores, in float32 throughout: float32 targets have no
// tensor-core path that keeps their precision (bf16 and tf32 operands drop 13 to 16 bits).
//
// A CTA of 256 threads holds 64 query rows and walks tiles of 64 slots: thread (ty, tx) of a
// 16 x 16 grid owns rows ty + 16 i and, of each tile's scores, slots tx + 16 j, then of the
// outputs four consecutive columns tx 4 + 64 j. Scores, the running maximum and sum, and the
// outputs stay in registers; keys, values and the tile's probabilities pass through shared
// memory, padded so that the 16 rows a warp reads at once fall into different banks.
#pragma once

#include "fe_attn_plan.cuh"

namespace fe {

constexpr int kSimtRows = 64, kSimtTile = 64, kSimtThreads = 256;
using SimtPlan = Plan<kSimtRows, kSimtTile, false, 1>;

template <int HD>
struct SimtSmem {
    static constexpr int kPad = HD + 4;
    float q[kSimtRows][kPad], k[kSimtTile][kPad], v[kSimtTile][HD], p[kSimtRows][kSimtTile + 4];
    int odd[2];  // the tile holds a non-finite value in a node's row (one flag per tile parity)
};

template <int HD>
__global__ void __launch_bounds__(kSimtThreads) tree_attn_simt_kernel(const __grid_constant__ TreeAttnArgs a) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    SimtSmem<HD>& sm = *reinterpret_cast<SimtSmem<HD>*>(smem_raw);
    const int t = threadIdx.x, tx = t & 15, ty = t >> 4;
    constexpr int NC = HD / 64;  // groups of four output columns per thread
    PlanArgs pa = plan_args(a);
    griddep_launch_dependents();
    bool bad = false;
    SegmentWalk<SimtPlan> walk;
    walk.init(pa, blockIdx.x, gridDim.x, &bad);
    if (bad && blockIdx.x == 0) atomicOr(a.status, ST_CAPACITY);
    const float scale2 = a.scale * kLog2e;
    if (t < 2) sm.odd[t] = 0;

    Segment g;
    bool any = false, continues = false;
    while (walk.next(pa, g)) {
        any = true;
        continues |= !g.whole && g.slot == 0;
        const int r0 = g.m * kSimtRows;
        __syncthreads();  // the previous segment's readers of sm.q are done
        for (int e = t; e < kSimtRows * HD; e += kSimtThreads) {
            const int r = e / HD, c = e % HD, row = r0 + r;
            float x = 0.f;
            if (row < g.rows) {
                const int node = row / a.G, head = g.h * a.G + row % a.G;
                x = ((const float*)a.q.p)[g.b * a.q.batch + node * a.q.token + head * a.q.head + c];
            }
            sm.q[r][c] = x * scale2;
        }
        float mx[4], sum[4], acc[4][NC][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            mx[i] = -INFINITY;
            sum[i] = 0.f;
#pragma unroll
            for (int j = 0; j < NC; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[i][j][k] = 0.f;
        }
        for (int tile = g.t0; tile < g.t1; ++tile) {
            const int par = tile & 1;
            __syncthreads();  // the previous tile's readers of k, v, p are done
            if (t == 0) sm.odd[par ^ 1] = 0;
            for (int e = t; e < kSimtTile * (HD / 4); e += kSimtThreads) {
                const int r = e / (HD / 4), c = e % (HD / 4) * 4;
                const int64_t slot = (int64_t)tile * kSimtTile + r;
                float4 kk = make_float4(0.f, 0.f, 0.f, 0.f), vv = kk;
                int64_t row;
                if (slot < g.end && cache_row(a.cache, g.b, slot, row, a.status)) {
                    row += g.h * head_step(a.cache);
                    kk = *reinterpret_cast<const float4*>((const float*)a.cache.k + row * HD + c);
                    vv = *reinterpret_cast<const float4*>((const float*)a.cache.v + row * HD + c);
                    if (slot >= g.s.P && !(finite_f32(vv.x) && finite_f32(vv.y) && finite_f32(vv.z) && finite_f32(vv.w)))
                        sm.odd[par] = 1;
                }
                *reinterpret_cast<float4*>(&sm.k[r][c]) = kk;
                *reinterpret_cast<float4*>(&sm.v[r][c]) = vv;
            }
            __syncthreads();
            float s[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
            for (int c = 0; c < HD; c += 4) {
                float4 q4[4], k4[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) q4[i] = *reinterpret_cast<const float4*>(&sm.q[ty + 16 * i][c]);
#pragma unroll
                for (int j = 0; j < 4; ++j) k4[j] = *reinterpret_cast<const float4*>(&sm.k[tx + 16 * j][c]);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[i][j] = fmaf(q4[i].x, k4[j].x, s[i][j]);
                        s[i][j] = fmaf(q4[i].y, k4[j].y, s[i][j]);
                        s[i][j] = fmaf(q4[i].z, k4[j].z, s[i][j]);
                        s[i][j] = fmaf(q4[i].w, k4[j].w, s[i][j]);
                    }
            }
            const bool odd = sm.odd[par] != 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int node = (r0 + ty + 16 * i) / a.G;
                bool see[4];
                float m = -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int slot = tile * kSimtTile + tx + 16 * j, c = slot - g.s.P;
                    see[j] = slot < g.end && node < g.s.n &&
                             (c < 0 || (a.mask ? a.mask[((int64_t)g.b * a.T + node) * a.T + c] != 0 : c <= node));
                    if (see[j]) m = fmaxf(m, s[i][j]);
                }
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                const float mn = fmaxf(mx[i], m), ms = mn == -INFINITY ? 0.f : mn;
                const float f = exp2f(mx[i] - ms);
                mx[i] = mn;
                float z = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float p = see[j] ? exp2f(s[i][j] - ms) : 0.f;
                    z += p;
                    // (-1 marks a hidden slot where a value row may hold infinities or NaN)
                    sm.p[ty + 16 * i][tx + 16 * j] = odd && !see[j] ? -1.f : p;
                }
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
                sum[i] = sum[i] * f + z;
#pragma unroll
                for (int j = 0; j < NC; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[i][j][k] *= f;
            }
            __syncwarp();  // a row's probabilities come from its own half warp
            if (!odd) {
#pragma unroll 4
                for (int c = 0; c < kSimtTile; ++c) {
                    float4 v4[NC];
#pragma unroll
                    for (int j = 0; j < NC; ++j) v4[j] = *reinterpret_cast<const float4*>(&sm.v[c][tx * 4 + 64 * j]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p = sm.p[ty + 16 * i][c];
#pragma unroll
                        for (int j = 0; j < NC; ++j) {
                            acc[i][j][0] = fmaf(p, v4[j].x, acc[i][j][0]);
                            acc[i][j][1] = fmaf(p, v4[j].y, acc[i][j][1]);
                            acc[i][j][2] = fmaf(p, v4[j].z, acc[i][j][2]);
                            acc[i][j][3] = fmaf(p, v4[j].w, acc[i][j][3]);
                        }
                    }
                }
            } else {
                for (int c = 0; c < kSimtTile; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p = sm.p[ty + 16 * i][c];
                        if (p == -1.f) continue;
#pragma unroll
                        for (int j = 0; j < NC; ++j)
#pragma unroll
                            for (int k = 0; k < 4; ++k) acc[i][j][k] = fmaf(p, sm.v[c][tx * 4 + 64 * j + k], acc[i][j][k]);
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = ty + 16 * i, row = r0 + r;
            if (row >= g.rows) continue;
            if (g.whole) {
                const int node = row / a.G, head = g.h * a.G + row % a.G;
                float* o = (float*)a.out.p + g.b * a.out.batch + node * a.out.token + head * a.out.head;
                const float inv = sum[i] == 0.f ? 0.f : 1.0f / sum[i];
#pragma unroll
                for (int j = 0; j < NC; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        o[tx * 4 + 64 * j + k] = sum[i] == 0.f ? 0.f : acc[i][j][k] * inv;
                if (a.lse && tx == 0)
                    a.lse[((int64_t)g.b * a.T + node) * a.H + head] =
                        sum[i] == 0.f ? -INFINITY : mx[i] * 0.6931471805599453f + logf(sum[i]);
            } else {
                const int64_t pr = ((int64_t)blockIdx.x * 2 + g.slot) * kAttnItemRows + r;
#pragma unroll
                for (int j = 0; j < NC; ++j)
                    *reinterpret_cast<float4*>(a.part_o + pr * HD + tx * 4 + 64 * j) =
                        make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
                if (tx == 0) {
                    a.part_ml[2 * pr] = mx[i];
                    a.part_ml[2 * pr + 1] = sum[i];
                }
            }
        }
    }
    if (t == 0) a.split[blockIdx.x] = walk.desc(pa, any, g, continues);
}

}  // namespace fe
