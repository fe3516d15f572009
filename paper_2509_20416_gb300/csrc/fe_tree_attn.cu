// Attention of a draft tree's nodes (or of consecutive tokens) over the cache
// (fe_tree_attention), and the join of items split between CTAs.
#include "fe_tree_attn_simt.cuh"
#include "fe_tree_attn_tc.cuh"

namespace fe {

namespace {

// ---- the join ------------------------------------------------------------------------------
// One warp per row (b, node, head): if the row's item was split, sum its partials in CTA order,
// sum_c 2^(m_c - m) (o_c, l_c) with m the largest m_c, and write the row; rows without any item
// (nodes past n_b) get zeros and -inf. Rows of whole items were written by the attention kernel.
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32;

template <typename QT, int HD, typename PL, int ROWS>
__global__ void __launch_bounds__(kJoinThreads) tree_attn_join_kernel(const __grid_constant__ TreeAttnArgs a, int ncta) {
    const PlanArgs pa = plan_args(a);
    const int lane = threadIdx.x & 31;
    const int b = blockIdx.y;
    // schedule: total units, and the first unit of this sequence (lengths are the caller's and
    // do not depend on the attention kernel, so this runs before the wait)
    int U = 0, before = 0;
#pragma unroll 1
    for (int bb = lane; bb < a.B; bb += 32) {
        const int u = PL::head_units(pa, seq_len(pa, bb)) * a.Hkv;
        U += u;
        if (bb < b) before += u;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        U += __shfl_xor_sync(0xffffffffu, U, o);
        before += __shfl_xor_sync(0xffffffffu, before, o);
    }
    const SeqLen s = seq_len(pa, b);
    const int rows = s.n * a.G;
    const int head_units = PL::head_units(pa, s);
    const Cut cut(U, ncta);
    griddep_wait();
    for (int x = blockIdx.x * kJoinWarps + threadIdx.x / 32; x < a.T * a.H; x += gridDim.x * kJoinWarps) {
        const int node = x / a.H, head = x % a.H, h = head / a.G;
        const int r = node * a.G + head % a.G;
        float o[HD / 32];
#pragma unroll
        for (int e = 0; e < HD / 32; ++e) o[e] = 0.f;
        float mx = -INFINITY, sum = 0.f;
        if (node < s.n) {
            const int m = r / ROWS, w = PL::weight(rows, m), nt = PL::tiles(pa, s, m);
            int s0 = before + h * head_units;
            if (pa.causal) {
#pragma unroll 1
                for (int k = 0; k < m; ++k) s0 += PL::tiles(pa, s, k) * PL::weight(rows, k);
            } else {
                s0 += m * nt * PL::weight(ROWS, 0);
            }
            const int c0 = cut.owner(s0), c1 = cut.owner(s0 + (nt - 1) * w);
            if (c0 == c1) continue;
            for (int c = c0; c <= c1; ++c) {
                const int u0 = cut.begin(c), u1 = cut.begin(c + 1);
                const int t0 = PL::first_tile(s0, w, nt, u0);
                if (t0 >= PL::first_tile(s0, w, nt, u1)) continue;  // no tile starts in this CTA's units
                const int64_t pr = ((int64_t)c * 2 + (t0 == 0 ? 1 : 0)) * kAttnItemRows + (r - m * ROWS);
                const float pm = __ldcg(a.part_ml + 2 * pr), pl = __ldcg(a.part_ml + 2 * pr + 1);
                const float* po = a.part_o + pr * HD + lane * (HD / 32);
                float v[HD / 32];
                if constexpr (HD == 128) {
                    const float4 f = __ldcg(reinterpret_cast<const float4*>(po));
                    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
                } else {
                    const float2 f = __ldcg(reinterpret_cast<const float2*>(po));
                    v[0] = f.x; v[1] = f.y;
                }
                const float mn = fmaxf(mx, pm), ms = mn == -INFINITY ? 0.f : mn;
                const float f0 = exp2f(mx - ms), f1 = exp2f(pm - ms);
                mx = mn;
                sum = sum * f0 + pl * f1;
#pragma unroll
                for (int e = 0; e < HD / 32; ++e) o[e] = o[e] * f0 + v[e] * f1;
            }
        }
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        QT* dst = (QT*)a.out.p + b * a.out.batch + node * a.out.token + head * a.out.head + lane * (HD / 32);
#pragma unroll
        for (int e = 0; e < HD / 32; ++e) store_one(dst + e, sum == 0.f ? 0.f : o[e] * inv);
        if (a.lse && lane == 0)
            a.lse[((int64_t)b * a.T + node) * a.H + head] =
                sum == 0.f ? -INFINITY : mx * 0.6931471805599453f + logf(sum);
    }
}

template <typename QT, int HD, typename PL, int ROWS>
cudaError_t launch_join(const TreeAttnArgs& a, int ncta, cudaStream_t st) {
    const int64_t rows = (int64_t)a.T * a.H;
    int64_t gx = (rows + kJoinWarps - 1) / kJoinWarps;
    const int64_t most = (152 * 8 + a.B - 1) / a.B;  // about one resident wave over all sequences
    if (gx > most) gx = most;
    return launch_k(tree_attn_join_kernel<QT, HD, PL, ROWS>, dim3((unsigned)gx, a.B), dim3(kJoinThreads), 0, st, true, a,
                    ncta);
}

template <int HD>
cudaError_t launch_simt(const TreeAttnArgs& a, int num_sms, cudaStream_t st) {
    const cudaError_t e = launch_k(tree_attn_simt_kernel<HD>, dim3(num_sms), dim3(kSimtThreads), sizeof(SimtSmem<HD>), st,
                                   false, a);
    if (e != cudaSuccess) return e;
    return launch_join<float, HD, SimtPlan, kSimtRows>(a, num_sms, st);
}

template <int HD, bool Q8, int MT>
cudaError_t launch_tc(const TreeAttnArgs& a, int num_sms, cudaStream_t st) {
    const cudaError_t e = launch_k(tree_attn_tc_kernel<HD, Q8, MT>, dim3(num_sms), dim3(TcShape<HD, Q8, MT>::kThreads),
                                   tc_smem<HD, Q8, MT>(), st, false, a);
    if (e != cudaSuccess) return e;
    return launch_join<bf16_t, HD, TcPlan, kAttnItemRows>(a, num_sms, st);
}

template <typename K>
cudaError_t allow_smem(K kern, size_t bytes) {
    return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <int HD>
cudaError_t prepare() {
    cudaError_t e;
    if ((e = allow_smem(tree_attn_simt_kernel<HD>, sizeof(SimtSmem<HD>))) != cudaSuccess) return e;
    if ((e = allow_smem(tree_attn_tc_kernel<HD, false, 1>, tc_smem<HD, false, 1>())) != cudaSuccess) return e;
    if ((e = allow_smem(tree_attn_tc_kernel<HD, false, 2>, tc_smem<HD, false, 2>())) != cudaSuccess) return e;
    if ((e = allow_smem(tree_attn_tc_kernel<HD, true, 1>, tc_smem<HD, true, 1>())) != cudaSuccess) return e;
    return allow_smem(tree_attn_tc_kernel<HD, true, 2>, tc_smem<HD, true, 2>());
}

template <int HD>
cudaError_t launch_hd(const TreeAttnArgs& a, fe_dtype dtype, fe_dtype cache_dtype, int num_sms, cudaStream_t st) {
    if (dtype == FE_F32) return launch_simt<HD>(a, num_sms, st);
    const bool one = (int64_t)a.T * a.G <= 128;  // every item fits one 128-row block: more tiles in flight
    if (cache_dtype == FE_E4M3)
        return one ? launch_tc<HD, true, 1>(a, num_sms, st) : launch_tc<HD, true, 2>(a, num_sms, st);
    return one ? launch_tc<HD, false, 1>(a, num_sms, st) : launch_tc<HD, false, 2>(a, num_sms, st);
}

}  // namespace

cudaError_t tree_attn_prepare() {
    const cudaError_t e = prepare<64>();
    return e != cudaSuccess ? e : prepare<128>();
}

bool tree_attn_fits(const TreeAttnArgs& a, fe_dtype dtype) {
    const int64_t rows = (int64_t)a.T * a.G;
    return dtype == FE_F32 ? SimtPlan::fits(a.B, a.Hkv, rows, a.cache.max_seq)
                           : TcPlan::fits(a.B, a.Hkv, rows, a.cache.max_seq);
}

cudaError_t launch_tree_attn(const TreeAttnArgs& a, fe_dtype dtype, fe_dtype cache_dtype, int hd, int num_sms,
                             cudaStream_t st) {
    return hd == 128 ? launch_hd<128>(a, dtype, cache_dtype, num_sms, st) : launch_hd<64>(a, dtype, cache_dtype, num_sms, st);
}

}  // namespace fe
