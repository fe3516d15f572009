// The join of attention items that were split between CTAs: sums the partial results of an item,
// sum_c 2^(m_c - m) (o_c, l_c) with m the largest m_c, in CTA order, and writes their rows; also
// fills the rows of nodes past n_b with zeros and -inf. At most one item begins in a CTA and goes on
// in the next: blocks x look at the one that attention CTA x noted (SplitDesc), blocks y share its
// rows and columns: a lane has 16 columns of a row, as the partials lie (four columns of a warp's 32
// rows are 512 bytes in a row). One pass, four contributors' reads under way at a time, the sums
// rescaled as their maximum grows. Bound by latency: its launch, which the attention's registers
// keep from overlapping, and two dependent reads (150 items of 196 rows: a row a warp took 20 us,
// this 8). A note never leads outside the workspace: an attention CTA clears its own before
// anything else, so that a CTA that gives up leaves none of an earlier call's, and the join looks no
// further than the grid's CTAs.
#pragma once

#include "fe_attn_plan.cuh"

namespace fe {

constexpr int kJoinThreads = 128, kJoinWarps = kJoinThreads / 32;

__device__ __forceinline__ void store_four(bf16_t* p, float a, float b, float c, float d, bool aligned) {
    const uint2 w = make_uint2(pack_bf16(a, b), pack_bf16(c, d));
    if (aligned) {
        *reinterpret_cast<uint2*>(p) = w;
    } else {
        p[0].bits = (uint16_t)w.x;
        p[1].bits = (uint16_t)(w.x >> 16);
        p[2].bits = (uint16_t)w.y;
        p[3].bits = (uint16_t)(w.y >> 16);
    }
}
__device__ __forceinline__ void store_four(float* p, float a, float b, float c, float d, bool aligned) {
    if (aligned) {
        *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
    } else {
        p[0] = a;
        p[1] = b;
        p[2] = c;
        p[3] = d;
    }
}

// Rows of sequence b's nodes from n on: zeros, -inf.
template <typename QT, int HD>
__device__ __forceinline__ void fill_rows(const TreeAttnArgs& a, int b, int n, int wid) {
    constexpr int E = HD / 32;
    const int lane = threadIdx.x & 31;
    for (int x = n * a.H + wid; x < a.T * a.H; x += gridDim.y * kJoinWarps) {
        QT* dst = (QT*)a.out.p + b * a.out.batch + (int64_t)(x / a.H) * a.out.token + (int64_t)(x % a.H) * a.out.head;
#pragma unroll
        for (int e = 0; e < E; ++e) store_one(dst + lane * E + e, 0.f);
        if (a.lse && lane == 0) a.lse[(int64_t)b * a.T * a.H + x] = -INFINITY;
    }
}

template <typename QT, int HD, int ROWS>
__global__ void __launch_bounds__(kJoinThreads) tree_attn_join_kernel(const __grid_constant__ TreeAttnArgs a) {
    const int lane = threadIdx.x & 31, wid = blockIdx.y * kJoinWarps + threadIdx.x / 32;
    griddep_wait();
    // rows of nodes past n_b
    if (a.nodes) {
        const PlanArgs pa = plan_args(a);
        for (int b = blockIdx.x; b < a.B; b += gridDim.x) fill_rows<QT, HD>(a, b, seq_len(pa, b).n, wid);
    } else {
        for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
            const int P = a.prefix[b];  // (a sequence out of range has no nodes)
            if (P < 0 || (int64_t)P + a.T > a.cache.max_seq) fill_rows<QT, HD>(a, b, 0, wid);
        }
    }
    const SplitDesc w = a.split[blockIdx.x];
    const int c0 = blockIdx.x, c1 = min(w.last, (int)gridDim.x - 1);
    if (c1 <= c0) return;
    const int r = wid / (HD / 16) * 32 + lane, col = wid % (HD / 16) * 16;
    if (r >= min(ROWS, w.rows - w.m * ROWS)) return;
    // contributor c's partial (a share of the item in which no tile starts has none: what lies there is
    // read all the same, ahead of the flag, and not used)
    auto slot = [&](int c) { return (int64_t)c * 2 + (c == c0 ? 1 : 0); };
    auto has = [&](int c) { return c == c0 || __ldcg(&a.split[c].has0) != 0; };
    float4 o[4];
    float mx = -INFINITY, sum = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int c = c0; c <= c1; ++c) {
        const float2 ml = __ldcg(reinterpret_cast<const float2*>(a.part_ml + 2 * (slot(c) * a.part_rows + r)));
        const float4* src = reinterpret_cast<const float4*>(a.part_o + slot(c) * a.part_rows * HD) + (int64_t)(col / 4) * a.part_rows + r;
        float4 v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __ldcg(src + e * a.part_rows);
        const bool mine = has(c);
        const float mn = mine ? fmaxf(mx, ml.x) : mx, ms = mn == -INFINITY ? 0.f : mn;
        const float f = exp2f(mx - ms), g = exp2f(ml.x - ms);
        mx = mn;
        if (!mine) continue;
        sum = sum * f + ml.y * g;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            o[e].x = o[e].x * f + v[e].x * g;
            o[e].y = o[e].y * f + v[e].y * g;
            o[e].z = o[e].z * f + v[e].z * g;
            o[e].w = o[e].w * f + v[e].w * g;
        }
    }
    const int row = w.m * ROWS + r, node = row / a.G, head = w.h * a.G + row % a.G;
    const bool none = sum == 0.f;
    const float inv = none ? 0.f : 1.0f / sum;
    QT* dst = (QT*)a.out.p + w.b * a.out.batch + (int64_t)node * a.out.token + (int64_t)head * a.out.head + col;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        store_four(dst + 4 * e, none ? 0.f : o[e].x * inv, none ? 0.f : o[e].y * inv, none ? 0.f : o[e].z * inv,
                   none ? 0.f : o[e].w * inv, a.out_vec);
    if (a.lse && col == 0)
        a.lse[((int64_t)w.b * a.T + node) * a.H + head] = none ? -INFINITY : mx * 0.6931471805599453f + logf(sum);
}

}  // namespace fe
