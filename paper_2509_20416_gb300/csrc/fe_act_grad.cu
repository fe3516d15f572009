// Gradients of activations, and sums over rows (fe_project_backward, fe_gated_ffn_backward): bound
// by memory traffic. A warp takes a strip of columns, 16 bytes a lane, of every eighth row of its
// CTA's part of the rows, so that a column's sum stays in a register until the part is done; the
// parts' sums are added in order by a second kernel. Measured (GB300): 4093 x 5120, bfloat16 gradient and float32
// pre-activation to bfloat16, with the sums, 30 us (5.6 TB/s); two rows of a warp in flight instead of four 58 us.
#include "fe_layer_common.cuh"

namespace fe {

namespace {

constexpr int kGradWarps = 8, kGradRows = 4;

// a row's columns of a lane, as loaded
template <typename T>
struct GradRow {
    uint4 d;
    float z[Vec16<T>::kN], u[Vec16<T>::kN];
};
template <typename T, bool FULL, bool GATED>
__device__ __forceinline__ void load_grad_row(const ActGradArgs& a, int64_t m, int n, int have, GradRow<T>& x) {
    constexpr int V = Vec16<T>::kN;
    const T* d = (const T*)a.dout.p + m * a.dout.row + n;
    if (FULL) {
        x.d = *reinterpret_cast<const uint4*>(d);
    } else {
        float f[V];
        load_row<T, V>(d, have, false, f);
        x.d = pack16<T>(f);
    }
    if (a.pre.p) load_row<float, V>((const float*)a.pre.p + m * a.pre.row + n, FULL ? V : have, FULL, x.z);
    if (GATED) load_row<float, V>((const float*)a.pre2.p + m * a.pre2.row + n, FULL ? V : have, FULL, x.u);
}

template <typename T, bool FULL, bool GATED>
__global__ void __launch_bounds__(kGradWarps * 32, 2) act_grad_kernel(const __grid_constant__ ActGradArgs a) {
    constexpr int V = Vec16<T>::kN;
    __shared__ float sums[kGradWarps][32][V + 1];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int n = (blockIdx.x * 32 + lane) * V, have = a.N - n;
    const int64_t r0 = (int64_t)a.part_rows * blockIdx.y, r1 = min(r0 + a.part_rows, a.M);
    float sum[V] = {};
    if (have > 0) {
        constexpr int F = GATED ? kGradRows / 2 : kGradRows;  // rows of a warp in flight
        for (int64_t r = r0 + warp; r < r1; r += F * kGradWarps) {
            GradRow<T> x[F];
#pragma unroll
            for (int f = 0; f < F; ++f)
                if (r + f * kGradWarps < r1) load_grad_row<T, FULL, GATED>(a, r + f * kGradWarps, n, have, x[f]);
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const int64_t m = r + f * kGradWarps;
                if (m >= r1) break;
                float d[V], e[V];
                Vec16<T>::widen(x[f].d, d);
                const float(&z)[V] = x[f].z, (&u)[V] = x[f].u;
                if (GATED) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        float v, dv;
                        act_both<kCoarse<T>>(a.act, z[i], v, dv);
                        e[i] = d[i] * v;
                        d[i] = d[i] * u[i] * dv;
                    }
                    store_row<T, V>((T*)a.d2.p + m * a.d2.row + n, FULL ? V : have, FULL, e);
                } else if (a.act != FE_ACT_NONE) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        float v, dv;
                        act_both<kCoarse<T>>(a.act, z[i], v, dv);
                        d[i] *= dv;
                    }
                }
                if (a.d1.p) store_row<T, V>((T*)a.d1.p + m * a.d1.row + n, FULL ? V : have, FULL, d);
#pragma unroll
                for (int i = 0; i < V; ++i) sum[i] += d[i];
            }
        }
    }
    if (!a.part) return;
#pragma unroll
    for (int i = 0; i < V; ++i) sums[warp][lane][i] = sum[i];
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * V; i += kGradWarps * 32) {
        const int c = blockIdx.x * 32 * V + i;
        if (c >= a.N) break;
        float s = 0.f;
        for (int w = 0; w < kGradWarps; ++w) s += sums[w][i / V][i % V];
        a.part[(int64_t)blockIdx.y * a.N + c] = s;
    }
}

// a warp's lanes take neighbouring columns, the warps of a CTA every 32nd part
constexpr int kSumWarps = 32;
template <typename T>
__global__ void __launch_bounds__(kSumWarps * 32) sum_parts_kernel(const __grid_constant__ SumJobs a) {
    __shared__ float sums[kSumWarps][32];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const SumJob& job = a.job[blockIdx.z];
    const int64_t c = (int64_t)blockIdx.x * 32 + lane, n = a.n;
    for (int64_t g = blockIdx.y; g < job.groups; g += gridDim.y) {
        float s = 0.f;
        if (c < n) {
            const float* p = job.part + g * job.parts * n + c;
#pragma unroll 8
            for (int64_t i = warp; i < job.parts; i += kSumWarps) s += p[i * n];
        }
        sums[warp][lane] = s;
        __syncthreads();
        if (warp == 0 && c < n) {
            s = 0.f;
#pragma unroll
            for (int w = 0; w < kSumWarps; ++w) s += sums[w][lane];
            store_one((T*)job.out + g * job.out_row + c, s);
        }
        __syncthreads();
    }
}

template <typename T>
cudaError_t launch_grad(const ActGradArgs& a, cudaStream_t st) {
    constexpr int V = Vec16<T>::kN, strip = 32 * V;
    const bool full = a.vec && a.N % V == 0;
    const auto kern = a.gated ? (full ? act_grad_kernel<T, true, true> : act_grad_kernel<T, false, true>)
                              : (full ? act_grad_kernel<T, true, false> : act_grad_kernel<T, false, false>);
    return launch_k(kern, dim3((a.N + strip - 1) / strip, a.parts), dim3(kGradWarps * 32), 0, st, false, a);
}

}  // namespace

// A part's rows fill its warps' turns; parts as many as give an SM some eight CTAs, within a grid's bounds.
void act_grad_plan(ActGradArgs& a, fe_dtype dtype, int num_sms) {
    const int strip = dtype == FE_F32 ? 128 : 256;
    const int64_t strips = (a.N + strip - 1) / strip, turn = kGradWarps * kGradRows, turns = (a.M + turn - 1) / turn;
    const int64_t want = (num_sms * 8 + strips - 1) / strips;
    int64_t k = (turns + want - 1) / want;
    a.part_rows = (int)(k * turn);
    a.parts = (int)((a.M + a.part_rows - 1) / a.part_rows);
}

cudaError_t launch_act_grad(const ActGradArgs& a, fe_dtype dtype, cudaStream_t st) {
    return dtype == FE_F32 ? launch_grad<float>(a, st) : launch_grad<bf16_t>(a, st);
}

cudaError_t launch_sum_parts(const SumJobs& a, fe_dtype dtype, cudaStream_t st) {
    int64_t groups = 1;
    for (int i = 0; i < a.jobs; ++i) groups = a.job[i].groups > groups ? a.job[i].groups : groups;
    if (!a.jobs) return cudaSuccess;
    const dim3 grid((unsigned)((a.n + 31) / 32), (unsigned)(groups < 65535 ? groups : 65535), a.jobs), block(kSumWarps * 32);
    return launch_k(dtype == FE_F32 ? sum_parts_kernel<float> : sum_parts_kernel<bf16_t>, grid, block, 0, st, false, a);
}

}  // namespace fe
