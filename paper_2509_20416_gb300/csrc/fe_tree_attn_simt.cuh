// Attention over the cache on the CUDA cores, in float32 throughout. (One bfloat16 or tf32 operand
// drops 13 to 16 bits; three bfloat16 parts a number, six products, would keep them on the tensor
// cores and have not been tried.)
//
// A CTA of 256 threads holds 16 NI query rows (NI = 1, 2 or 4, the fewest that hold an item's) and
// walks tiles of 64 slots: thread (ty, tx) of a 16 x 16 grid owns rows ty + 16 i and, of each tile's
// scores, slots tx + 16 j, then of the outputs four consecutive columns tx 4 + 64 j. Scores, the
// running maximum and sum, and the outputs stay in registers; keys, values and the tile's
// probabilities pass through shared memory, padded so that the 16 rows a warp reads at once fall
// into different banks. Meanwhile the next tile's rows arrive (cp.async) in a second buffer, or,
// where two CTAs fit an SM only with one buffer, the other CTA works. Products go two columns to an
// instruction (packed float32 pairs). With 64 rows bound by shared memory: a tile of 128-wide heads
// needs 8192 clocks of products and takes 22 thousand, as a warp gets its 16-byte operands at 4 clocks a load,
// eight loads for 64 products of a thread; with 16 rows by the same and by latency.
// Fewer rows take fewer operations and leave room for the second CTA: 32 sequences over 256 to 4096
// slots, 128-wide heads, 16 rows an item: 467 us with 64 rows a CTA, 357 with 16; 36 rows (64 a CTA)
// 631 us, 16 TFLOP/s. 64-wide heads, one CTA an SM or two: 402 or 320 us at 36 rows, 22 or 24 us for
// 16 short items.
#pragma once

#include "fe_attn_plan.cuh"

namespace fe {

constexpr int kSimtThreads = 256;
template <int HD, int NI>
struct SimtSmem {
    static constexpr int kPad = HD + 4;
    static constexpr int kBufs = HD == 128 && NI <= 2 ? 1 : 2, kCtas = HD == 128 && NI == 4 ? 1 : 2;  // CTAs an SM
    float q[16 * NI][kPad], k[kBufs][kSimtTile][kPad], v[kBufs][kSimtTile][HD], p[16 * NI][kSimtTile + 4];
    int odd[2];  // by the tile's parity in the walk: it holds a non-finite value in a node's row
};

template <int HD, int NI>
__global__ void __launch_bounds__(kSimtThreads, SimtSmem<HD, NI>::kCtas) tree_attn_simt_kernel(const __grid_constant__ TreeAttnArgs a) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    SimtSmem<HD, NI>& sm = *reinterpret_cast<SimtSmem<HD, NI>*>(smem_raw);
    const int t = threadIdx.x, tx = t & 15, ty = t >> 4;
    constexpr int NC = HD / 64;  // groups of four output columns per thread
    constexpr bool kTwo = SimtSmem<HD, NI>::kBufs == 2;
    PlanArgs pa = plan_args(a);
    griddep_launch_dependents();
    bool bad = false;
    SegmentWalk<SimtPlan<NI>> walk;
    walk.init(pa, blockIdx.x, gridDim.x, &bad);
    if (bad && blockIdx.x == 0) atomicOr(a.status, ST_CAPACITY);
    const float scale2 = a.scale * kLog2e;
    if (t < 2) sm.odd[t] = 0;
    __syncthreads();

    Segment g;
    bool any = false, continues = false;
    int buf = 0, par = 0;
    while (walk.next(pa, g)) {
        any = true;
        continues |= !g.whole && g.slot == 0;
        const int r0 = g.m * 16 * NI;
        // a thread's 16-byte chunks of a tile's keys and values, into buffer `to`
        auto load = [&](int tile, int to) {
#pragma unroll 1
            for (int e = t; e < kSimtTile * (HD / 4); e += kSimtThreads) {
                const int r = e / (HD / 4), c = e % (HD / 4) * 4;
                const int64_t slot = (int64_t)tile * kSimtTile + r;
                int64_t row = 0;
                const bool ok = slot < g.end && cache_row(a.cache, g.b, slot, row, a.status);
                if (ok) row += g.h * head_step(a.cache);
                cp_async16(smem_u32(&sm.k[to][r][c]), (const float*)a.cache.k + row * HD + c, ok);
                cp_async16(smem_u32(&sm.v[to][r][c]), (const float*)a.cache.v + row * HD + c, ok);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        if (kTwo) load(g.t0, buf);  // (the last reads of sm were before the barrier that ended the last tile)
        for (int e = t; e < 16 * NI * HD; e += kSimtThreads) {
            const int r = e / HD, c = e % HD, row = r0 + r;
            float x = 0.f;
            if (row < g.rows) {
                const int node = row / a.G, head = g.h * a.G + row % a.G;
                x = ((const float*)a.q.p)[g.b * a.q.batch + node * a.q.token + head * a.q.head + c];
            }
            sm.q[r][c] = x * scale2;
        }
        float mx[NI], sum[NI];
        uint64_t acc[NI][NC][2];  // pairs of columns
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            mx[i] = -INFINITY;
            sum[i] = 0.f;
#pragma unroll
            for (int j = 0; j < NC; ++j)
#pragma unroll
                for (int k = 0; k < 2; ++k) acc[i][j][k] = 0;
        }
        for (int tile = g.t0; tile < g.t1; ++tile, buf ^= kTwo, par ^= 1) {
            if (kTwo && tile + 1 < g.t1) {
                load(tile + 1, buf ^ 1);
                asm volatile("cp.async.wait_group 1;" ::: "memory");
            } else {
                if (!kTwo) load(tile, buf);
                asm volatile("cp.async.wait_group 0;" ::: "memory");
            }
            if ((tile + 1) * kSimtTile > g.s.P) {  // the thread's own chunks of nodes' value rows
#pragma unroll 1
                for (int e = t; e < kSimtTile * (HD / 4); e += kSimtThreads) {
                    const int r = e / (HD / 4), c = e % (HD / 4) * 4;
                    const float4 x = *reinterpret_cast<const float4*>(&sm.v[buf][r][c]);
                    if (tile * kSimtTile + r >= g.s.P && !(finite_f32(x.x) && finite_f32(x.y) && finite_f32(x.z) && finite_f32(x.w)))
                        sm.odd[par] = 1;
                }
            }
            __syncthreads();
            float s[NI][4];
            {
                uint64_t s2[NI][4];  // even and odd columns' sums
#pragma unroll
                for (int i = 0; i < NI; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s2[i][j] = 0;
#pragma unroll 4
                for (int c = 0; c < HD; c += 4) {
                    ulonglong2 q4[NI], k4[4];
#pragma unroll
                    for (int i = 0; i < NI; ++i) q4[i] = *reinterpret_cast<const ulonglong2*>(&sm.q[ty + 16 * i][c]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) k4[j] = *reinterpret_cast<const ulonglong2*>(&sm.k[buf][tx + 16 * j][c]);
#pragma unroll
                    for (int i = 0; i < NI; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) s2[i][j] = fma_x2(q4[i].y, k4[j].y, fma_x2(q4[i].x, k4[j].x, s2[i][j]));
                }
#pragma unroll
                for (int i = 0; i < NI; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[i][j] = low_f32(s2[i][j]) + high_f32(s2[i][j]);
            }
            const bool odd = sm.odd[par] != 0;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
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
                    for (int k = 0; k < 2; ++k) acc[i][j][k] = mul_x2(acc[i][j][k], pair_f32(f));
            }
            __syncwarp();  // a row's probabilities come from its own half warp
            if (!odd) {
#pragma unroll 2
                for (int c = 0; c < kSimtTile; c += 4) {
                    float4 p4[NI];
#pragma unroll
                    for (int i = 0; i < NI; ++i) p4[i] = *reinterpret_cast<const float4*>(&sm.p[ty + 16 * i][c]);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        ulonglong2 v4[NC];
#pragma unroll
                        for (int j = 0; j < NC; ++j) v4[j] = *reinterpret_cast<const ulonglong2*>(&sm.v[buf][c + u][tx * 4 + 64 * j]);
#pragma unroll
                        for (int i = 0; i < NI; ++i) {
                            const uint64_t p = pair_f32(u == 0 ? p4[i].x : u == 1 ? p4[i].y : u == 2 ? p4[i].z : p4[i].w);
#pragma unroll
                            for (int j = 0; j < NC; ++j) {
                                acc[i][j][0] = fma_x2(p, v4[j].x, acc[i][j][0]);
                                acc[i][j][1] = fma_x2(p, v4[j].y, acc[i][j][1]);
                            }
                        }
                    }
                }
            } else {
                for (int c = 0; c < kSimtTile; ++c)
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
                        const float p = sm.p[ty + 16 * i][c];
                        if (p == -1.f) continue;
#pragma unroll
                        for (int j = 0; j < NC; ++j)
#pragma unroll
                            for (int k = 0; k < 2; ++k)
                                acc[i][j][k] = fma_x2(pair_f32(p), *reinterpret_cast<const uint64_t*>(&sm.v[buf][c][tx * 4 + 64 * j + 2 * k]), acc[i][j][k]);
                    }
            }
            __syncthreads();  // this buffer's (and p's) readers are done
            if (t == 0) sm.odd[par] = 0;  // (set again two tiles on, a barrier later)
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
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
                        o[tx * 4 + 64 * j + k] = sum[i] == 0.f ? 0.f : (k & 1 ? high_f32(acc[i][j][k / 2]) : low_f32(acc[i][j][k / 2])) * inv;
                if (a.lse && tx == 0)
                    a.lse[((int64_t)g.b * a.T + node) * a.H + head] =
                        sum[i] == 0.f ? -INFINITY : mx[i] * 0.6931471805599453f + logf(sum[i]);
            } else {
                const int64_t pr = ((int64_t)blockIdx.x * 2 + g.slot) * a.part_rows + r;
#pragma unroll
                for (int j = 0; j < NC; ++j)
                    *reinterpret_cast<float4*>(a.part_o + (pr - r) * HD + ((tx + 16 * j) * a.part_rows + r) * 4) =
                        make_float4(low_f32(acc[i][j][0]), high_f32(acc[i][j][0]), low_f32(acc[i][j][1]), high_f32(acc[i][j][1]));
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
