// The norms behind a block and before the next with the block's gate and residual (fe_block_norm),
// and their gradient. Bound by memory traffic: a row's vectors are read once, stay in registers for
// the statistics that depend on one another, and are written once.
//
//   forward   p = z rz (w_post + o), y = x + s g p, n = y ry (w_pre + o), r = 1 / sqrt(mean of squares + eps)
//   backward  with a = dn (w_pre + o):
//             dx = dy + ry a - y ry^3 mean(a y)
//             dp = s g dx, b = dp (w_post + o):  dz = rz b - z rz^3 mean(b z)
//             dw_pre = sum dn y ry,  dw_post = sum dp z rz,  dg = sum s p dx
//             (y is computed again from x and z, so nothing rounded stands in for it)
//
// A worker is a CTA, or a warp where a row is at most 32 vectors of 16 bytes; its threads own
// columns, so that the sums over rows stay in registers. The next row's loads are in flight while
// a row's statistics are reduced.
#include "fe_layer_common.cuh"

namespace fe {

namespace {

template <typename T>
__device__ __forceinline__ uint4 load_raw(const void* base, int64_t at, int have, bool vec) {
    constexpr int V = Vec16<T>::kN;
    const T* p = (const T*)base + at;
    if (vec && have >= V) return *reinterpret_cast<const uint4*>(p);
    float f[V];
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = i < have ? load_one(p + i) : 0.f;
    return pack16<T>(f);
}

// N sums over a worker's threads at once; buf: two halves that calls take in turn
template <bool WARP, int N>
__device__ __forceinline__ void worker_sum(float* v, float (*buf)[32 * 2], int& turn) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
    if (WARP) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    float* b = buf[turn];
    turn ^= 1;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) b[i * 32 + warp] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(lane < warps ? b[i * 32 + lane] : 0.f);
}

// w + offset for a thread's columns; 1 without weights
template <typename T>
__device__ __forceinline__ void weights(const void* w, int c, int have, bool vec, float offset, float* f) {
    constexpr int V = Vec16<T>::kN;
    if (!w) {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = 1.f;
        return;
    }
    load_row<T, V>((const T*)w + c, have, vec, f);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] += offset;
}

template <typename T, int VPT, bool WARP, int MAXT>
__global__ void __launch_bounds__(MAXT) norm_kernel(const __grid_constant__ NormArgs a) {
    constexpr int V = Vec16<T>::kN;
    __shared__ float buf[2][64];
    int turn = 0;
    const int nt = WARP ? 32 : blockDim.x, tid = WARP ? threadIdx.x % 32 : threadIdx.x;
    const int64_t step = WARP ? (int64_t)gridDim.x * (blockDim.x / 32) : gridDim.x;
    int64_t r = WARP ? (int64_t)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32 : blockIdx.x;
    const float inv_d = 1.f / (float)a.d;
    uint4 rx[VPT], rz[VPT];
    const auto fetch = [&](int64_t row) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = (j * nt + tid) * V, have = a.d - c;
            if (have <= 0) {
                rx[j] = rz[j] = make_uint4(0, 0, 0, 0);
                continue;
            }
            rx[j] = load_raw<T>(a.x.p, row * a.x.row + c, have, a.vec);
            if (a.z.p) rz[j] = load_raw<T>(a.z.p, row * a.z.row + c, have, a.vec);
        }
    };
    if (r < a.R) fetch(r);
    for (; r < a.R; r += step) {
        float y[VPT][V];
        float scale_z = 1.f;
        if (a.post) {
            float s[1] = {0.f};
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                float z[V];
                Vec16<T>::widen(rz[j], z);
#pragma unroll
                for (int i = 0; i < V; ++i) s[0] += z[i] * z[i];
            }
            worker_sum<WARP, 1>(s, buf, turn);
            scale_z = rsqrtf(s[0] * inv_d + a.eps);
        }
        float s[1] = {0.f};
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = (j * nt + tid) * V, have = a.d - c;
            Vec16<T>::widen(rx[j], y[j]);
            if (have > 0 && a.z.p) {
                float z[V], w[V];
                Vec16<T>::widen(rz[j], z);
                if (a.post) {
                    weights<T>(a.post_w, c, have, a.vec, a.offset, w);
#pragma unroll
                    for (int i = 0; i < V; ++i) z[i] *= scale_z * w[i];
                }
                if (a.gate.p) {
                    load_row<T, V>((const T*)a.gate.p + r / a.gate_rows * a.gate.row + c, have, a.vec, w);
#pragma unroll
                    for (int i = 0; i < V; ++i) z[i] *= w[i];
                }
#pragma unroll
                for (int i = 0; i < V; ++i) y[j][i] = fmaf(a.scale, z[i], y[j][i]);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += y[j][i] * y[j][i];
        }
        if (r + step < a.R) fetch(r + step);  // (a row is never both: outputs may be the inputs themselves)
        if (a.y.p) {
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int c = (j * nt + tid) * V;
                store_row<T, V>((T*)a.y.p + r * a.y.row + c, a.d - c, a.vec, y[j]);
            }
        }
        if (!a.n.p) continue;
        worker_sum<WARP, 1>(s, buf, turn);
        const float scale_y = rsqrtf(s[0] * inv_d + a.eps);
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = (j * nt + tid) * V, have = a.d - c;
            if (have <= 0) continue;
            float w[V];
            weights<T>(a.pre_w, c, have, a.vec, a.offset, w);
#pragma unroll
            for (int i = 0; i < V; ++i) w[i] *= y[j][i] * scale_y;
            store_row<T, V>((T*)a.n.p + r * a.n.row + c, have, a.vec, w);
        }
    }
}

// Rows of any length: the statistics in passes of their own over the row (which the caches hold).
template <typename T>
__global__ void __launch_bounds__(1024) norm_long_kernel(const __grid_constant__ NormArgs a) {
    constexpr int V = Vec16<T>::kN;
    __shared__ float buf[2][64];
    int turn = 0;
    const float inv_d = 1.f / (float)a.d;
    for (int64_t r = blockIdx.x; r < a.R; r += gridDim.x) {
        float scale_z = 1.f, s[1] = {0.f};
        if (a.post) {
            for (int c = threadIdx.x * V; c < a.d; c += blockDim.x * V) {
                float z[V];
                load_row<T, V>((const T*)a.z.p + r * a.z.row + c, a.d - c, a.vec, z);
#pragma unroll
                for (int i = 0; i < V; ++i) s[0] += z[i] * z[i];
            }
            worker_sum<false, 1>(s, buf, turn);
            scale_z = rsqrtf(s[0] * inv_d + a.eps);
        }
        const auto row_y = [&](int c, int have, float* y) {
            load_row<T, V>((const T*)a.x.p + r * a.x.row + c, have, a.vec, y);
            if (!a.z.p) return;
            float z[V], w[V];
            load_row<T, V>((const T*)a.z.p + r * a.z.row + c, have, a.vec, z);
            if (a.post) {
                weights<T>(a.post_w, c, have, a.vec, a.offset, w);
#pragma unroll
                for (int i = 0; i < V; ++i) z[i] *= scale_z * w[i];
            }
            if (a.gate.p) {
                load_row<T, V>((const T*)a.gate.p + r / a.gate_rows * a.gate.row + c, have, a.vec, w);
#pragma unroll
                for (int i = 0; i < V; ++i) z[i] *= w[i];
            }
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = fmaf(a.scale, z[i], y[i]);
        };
        float scale_y = 0.f;
        if (a.n.p) {
            s[0] = 0.f;
            for (int c = threadIdx.x * V; c < a.d; c += blockDim.x * V) {
                float y[V];
                row_y(c, a.d - c, y);
#pragma unroll
                for (int i = 0; i < V; ++i) s[0] += y[i] * y[i];
            }
            worker_sum<false, 1>(s, buf, turn);
            scale_y = rsqrtf(s[0] * inv_d + a.eps);
        }
        for (int c = threadIdx.x * V; c < a.d; c += blockDim.x * V) {
            const int have = a.d - c;
            float y[V], w[V];
            row_y(c, have, y);
            if (a.y.p) store_row<T, V>((T*)a.y.p + r * a.y.row + c, have, a.vec, y);
            if (!a.n.p) continue;
            weights<T>(a.pre_w, c, have, a.vec, a.offset, w);
#pragma unroll
            for (int i = 0; i < V; ++i) w[i] *= y[i] * scale_y;
            store_row<T, V>((T*)a.n.p + r * a.n.row + c, have, a.vec, w);
        }
    }
}

// the rows of worker w: of one group's part, or of whole groups
__device__ __forceinline__ void worker_rows(const NormArgs& a, int64_t w, int64_t& r0, int64_t& r1) {
    const int64_t size = a.gate.p ? a.gate_rows : a.R;
    if (a.parts) {
        const int64_t g = w / a.parts, p = w % a.parts, first = g * size, len = min(size, a.R - first);
        r0 = first + len * p / a.parts;
        r1 = first + len * (p + 1) / a.parts;
    } else {
        r0 = min(w * a.step * size, a.R);
        r1 = min((w + 1) * a.step * size, a.R);
    }
}

template <typename T, int VPT, bool WARP, int MAXT>
__global__ void __launch_bounds__(MAXT) norm_backward_kernel(const __grid_constant__ NormArgs a, int64_t workers) {
    constexpr int V = Vec16<T>::kN;
    __shared__ float buf[2][64];
    int turn = 0;
    const int nt = WARP ? 32 : blockDim.x, tid = WARP ? threadIdx.x % 32 : threadIdx.x;
    const int64_t worker = WARP ? (int64_t)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32 : blockIdx.x;
    if (worker >= workers) return;  // (a whole warp, where warps are workers)
    const float inv_d = 1.f / (float)a.d;
    int64_t r, r1;
    worker_rows(a, worker, r, r1);
    uint4 rx[VPT], rz[VPT], ry[VPT], rn[VPT];
    const auto fetch = [&](int64_t row) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = (j * nt + tid) * V, have = a.d - c;
            rx[j] = rz[j] = ry[j] = rn[j] = make_uint4(0, 0, 0, 0);
            if (have <= 0) continue;
            rx[j] = load_raw<T>(a.x.p, row * a.x.row + c, have, a.vec);
            if (a.z.p) rz[j] = load_raw<T>(a.z.p, row * a.z.row + c, have, a.vec);
            if (a.dy.p) ry[j] = load_raw<T>(a.dy.p, row * a.dy.row + c, have, a.vec);
            if (a.dn.p) rn[j] = load_raw<T>(a.dn.p, row * a.dn.row + c, have, a.vec);
        }
    };
    float spre[VPT][V] = {}, spost[VPT][V] = {}, sgate[VPT][V] = {};
    int64_t group = 0, group_end = a.R;  // rows of the current gate
    if (a.gate.p) {
        group = r / a.gate_rows;
        group_end = (group + 1) * a.gate_rows;
    }
    if (r < r1) fetch(r);
    for (; r < r1; ++r) {
        float scale_z = 1.f;
        if (a.post) {
            float s[1] = {0.f};
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                float z[V];
                Vec16<T>::widen(rz[j], z);
#pragma unroll
                for (int i = 0; i < V; ++i) s[0] += z[i] * z[i];
            }
            worker_sum<WARP, 1>(s, buf, turn);
            scale_z = rsqrtf(s[0] * inv_d + a.eps);
        }
        // y (in dx's place), p and a = dn (w_pre + o)
        float y[VPT][V], p[VPT][V], dn[VPT][V], t[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = (j * nt + tid) * V, have = a.d - c;
            float w[V];
            Vec16<T>::widen(rx[j], y[j]);
            Vec16<T>::widen(rz[j], p[j]);
            Vec16<T>::widen(rn[j], dn[j]);
            if (have > 0 && a.z.p) {
                if (a.post) {
                    weights<T>(a.post_w, c, have, a.vec, a.offset, w);
#pragma unroll
                    for (int i = 0; i < V; ++i) p[j][i] *= scale_z * w[i];
                }
#pragma unroll
                for (int i = 0; i < V; ++i) w[i] = 1.f;
                if (a.gate.p) load_row<T, V>((const T*)a.gate.p + group * a.gate.row + c, have, a.vec, w);
#pragma unroll
                for (int i = 0; i < V; ++i) y[j][i] = fmaf(a.scale, p[j][i] * w[i], y[j][i]);
            }
            if (have > 0 && a.dn.p) {
                weights<T>(a.pre_w, c, have, a.vec, a.offset, w);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    t[0] += y[j][i] * y[j][i];
                    t[1] += dn[j][i] * w[i] * y[j][i];
                }
            }
        }
        float scale_y = 0.f, back = 0.f;
        if (a.dn.p) {
            worker_sum<WARP, 2>(t, buf, turn);
            scale_y = rsqrtf(t[0] * inv_d + a.eps);
            back = t[1] * inv_d * scale_y * scale_y * scale_y;
        }
        float u[1] = {0.f};
        float dp[VPT][V];
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = (j * nt + tid) * V, have = a.d - c;
            float w[V], dx[V];
            Vec16<T>::widen(ry[j], dx);
            if (have <= 0) continue;
            if (a.dn.p) {
                weights<T>(a.pre_w, c, have, a.vec, a.offset, w);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    dx[i] += scale_y * dn[j][i] * w[i] - back * y[j][i];
                    spre[j][i] = fmaf(dn[j][i], y[j][i] * scale_y, spre[j][i]);
                }
            }
            if (a.dx.p) store_row<T, V>((T*)a.dx.p + r * a.dx.row + c, have, a.vec, dx);
            if (!a.z.p) continue;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                dp[j][i] = a.scale * dx[i];
                sgate[j][i] = fmaf(dp[j][i], p[j][i], sgate[j][i]);
            }
            if (a.gate.p) {
                load_row<T, V>((const T*)a.gate.p + group * a.gate.row + c, have, a.vec, w);
#pragma unroll
                for (int i = 0; i < V; ++i) dp[j][i] *= w[i];
            }
            if (a.post) {
                float z[V];
                Vec16<T>::widen(rz[j], z);
                weights<T>(a.post_w, c, have, a.vec, a.offset, w);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    spost[j][i] = fmaf(dp[j][i], z[i] * scale_z, spost[j][i]);
                    dp[j][i] *= w[i];
                    u[0] += dp[j][i] * z[i];
                    p[j][i] = z[i];  // (p has been used)
                }
            }
        }
        if (r + 1 < r1) fetch(r + 1);
        if (a.post) worker_sum<WARP, 1>(u, buf, turn);
        if (a.dz.p) {
            const float back_z = u[0] * inv_d * scale_z * scale_z * scale_z;
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int c = (j * nt + tid) * V, have = a.d - c;
                if (have <= 0) continue;
                if (a.post) {
#pragma unroll
                    for (int i = 0; i < V; ++i) dp[j][i] = scale_z * dp[j][i] - back_z * p[j][i];
                }
                store_row<T, V>((T*)a.dz.p + r * a.dz.row + c, have, a.vec, dp[j]);
            }
        }
        if (r + 1 == group_end || (r + 1 == r1 && !a.parts)) {  // the last row of a gate
            if (a.dgate.p && !a.part_gate) {
#pragma unroll
                for (int j = 0; j < VPT; ++j) {
                    const int c = (j * nt + tid) * V;
                    store_row<T, V>((T*)a.dgate.p + group * a.dgate.row + c, a.d - c, a.vec, sgate[j]);
#pragma unroll
                    for (int i = 0; i < V; ++i) sgate[j][i] = 0.f;
                }
            }
            if (a.gate.p) {
                ++group;
                group_end += a.gate_rows;
            }
        }
    }
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int c = (j * nt + tid) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (c + i >= a.d) continue;
            if (a.part_pre) a.part_pre[worker * a.d + c + i] = spre[j][i];
            if (a.part_post) a.part_post[worker * a.d + c + i] = spost[j][i];
            if (a.part_gate) a.part_gate[worker * a.d + c + i] = sgate[j][i];
        }
    }
}

// Rows of any length: passes over the row, the sums over rows in the worker's own part of memory.
template <typename T>
__global__ void __launch_bounds__(1024) norm_backward_long_kernel(const __grid_constant__ NormArgs a) {
    constexpr int V = Vec16<T>::kN;
    __shared__ float buf[2][64];
    int turn = 0;
    const int64_t worker = blockIdx.x;
    const float inv_d = 1.f / (float)a.d;
    int64_t r0, r1;
    worker_rows(a, worker, r0, r1);
    float* const ppre = a.part_pre ? a.part_pre + worker * a.d : nullptr;
    float* const ppost = a.part_post ? a.part_post + worker * a.d : nullptr;
    float* const pgate = a.part_gate ? a.part_gate + worker * a.d : nullptr;
    for (int c = threadIdx.x * V; c < a.d; c += blockDim.x * V)
        for (int i = 0; i < V && c + i < a.d; ++i) {
            if (ppre) ppre[c + i] = 0.f;
            if (ppost) ppost[c + i] = 0.f;
            if (pgate) pgate[c + i] = 0.f;
        }
    for (int64_t r = r0; r < r1; ++r) {
        const int64_t group = a.gate.p ? r / a.gate_rows : 0;
        const bool first = a.gate.p && r % a.gate_rows == 0, last = a.gate.p && (r + 1 == a.R || (r + 1) % a.gate_rows == 0);
        float scale_z = 1.f, s[1] = {0.f};
        if (a.post) {
            for (int c = threadIdx.x * V; c < a.d; c += blockDim.x * V) {
                float z[V];
                load_row<T, V>((const T*)a.z.p + r * a.z.row + c, a.d - c, a.vec, z);
#pragma unroll
                for (int i = 0; i < V; ++i) s[0] += z[i] * z[i];
            }
            worker_sum<false, 1>(s, buf, turn);
            scale_z = rsqrtf(s[0] * inv_d + a.eps);
        }
        // y, p, z and the gate of a thread's columns
        const auto row = [&](int c, int have, float* y, float* p, float* z, float* g) {
            load_row<T, V>((const T*)a.x.p + r * a.x.row + c, have, a.vec, y);
#pragma unroll
            for (int i = 0; i < V; ++i) p[i] = z[i] = 0.f, g[i] = 1.f;
            if (!a.z.p) return;
            load_row<T, V>((const T*)a.z.p + r * a.z.row + c, have, a.vec, z);
            float w[V];
            if (a.post) weights<T>(a.post_w, c, have, a.vec, a.offset, w);
            if (a.gate.p) load_row<T, V>((const T*)a.gate.p + group * a.gate.row + c, have, a.vec, g);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                p[i] = a.post ? z[i] * (scale_z * w[i]) : z[i];
                y[i] = fmaf(a.scale, p[i] * g[i], y[i]);
            }
        };
        float t[2] = {0.f, 0.f}, scale_y = 0.f, back = 0.f;
        float y[V], p[V], z[V], g[V], w[V], dn[V], dx[V];
        if (a.dn.p) {
            for (int c = threadIdx.x * V; c < a.d; c += blockDim.x * V) {
                const int have = a.d - c;
                row(c, have, y, p, z, g);
                load_row<T, V>((const T*)a.dn.p + r * a.dn.row + c, have, a.vec, dn);
                weights<T>(a.pre_w, c, have, a.vec, a.offset, w);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    t[0] += y[i] * y[i];
                    t[1] += dn[i] * w[i] * y[i];
                }
            }
            worker_sum<false, 2>(t, buf, turn);
            scale_y = rsqrtf(t[0] * inv_d + a.eps);
            back = t[1] * inv_d * scale_y * scale_y * scale_y;
        }
        const auto row_dx = [&](int c, int have) {
#pragma unroll
            for (int i = 0; i < V; ++i) dx[i] = 0.f;
            if (a.dy.p) load_row<T, V>((const T*)a.dy.p + r * a.dy.row + c, have, a.vec, dx);
            if (!a.dn.p) return;
            load_row<T, V>((const T*)a.dn.p + r * a.dn.row + c, have, a.vec, dn);
            weights<T>(a.pre_w, c, have, a.vec, a.offset, w);
#pragma unroll
            for (int i = 0; i < V; ++i) dx[i] += scale_y * dn[i] * w[i] - back * y[i];
        };
        float u[1] = {0.f};
        if (a.post) {
            for (int c = threadIdx.x * V; c < a.d; c += blockDim.x * V) {
                row(c, a.d - c, y, p, z, g);
                row_dx(c, a.d - c);
                weights<T>(a.post_w, c, a.d - c, a.vec, a.offset, w);
#pragma unroll
                for (int i = 0; i < V; ++i) u[0] += a.scale * dx[i] * g[i] * w[i] * z[i];
            }
            worker_sum<false, 1>(u, buf, turn);
        }
        const float back_z = u[0] * inv_d * scale_z * scale_z * scale_z;
        for (int c = threadIdx.x * V; c < a.d; c += blockDim.x * V) {
            const int have = a.d - c;
            row(c, have, y, p, z, g);
            row_dx(c, have);
            if (ppre && a.dn.p) {
                for (int i = 0; i < V && i < have; ++i) ppre[c + i] += dn[i] * (y[i] * scale_y);
            }
            if (a.dx.p) store_row<T, V>((T*)a.dx.p + r * a.dx.row + c, have, a.vec, dx);
            if (!a.z.p) continue;
            if (pgate) {
                for (int i = 0; i < V && i < have; ++i) {
                    const float v = (first && !a.parts ? 0.f : pgate[c + i]) + a.scale * dx[i] * p[i];
                    pgate[c + i] = v;
                    if (last && !a.parts) store_one((T*)a.dgate.p + group * a.dgate.row + c + i, v);
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) dx[i] *= a.scale * g[i];
            if (a.post) {
                if (ppost) {
                    for (int i = 0; i < V && i < have; ++i) ppost[c + i] += dx[i] * (z[i] * scale_z);
                }
                weights<T>(a.post_w, c, have, a.vec, a.offset, w);
#pragma unroll
                for (int i = 0; i < V; ++i) dx[i] = scale_z * dx[i] * w[i] - back_z * z[i];
            }
            if (a.dz.p) store_row<T, V>((T*)a.dz.p + r * a.dz.row + c, have, a.vec, dx);
        }
    }
}

// threads of a CTA for a row of nv vectors, VPT a thread
int cta_threads(int64_t nv, int vpt) { return (int)(((nv + vpt - 1) / vpt + 31) / 32 * 32); }

template <typename K>
cudaError_t resident(K kern, int threads, int num_sms, int64_t rows, unsigned& grid) {
    int per = 0;
    const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kern, threads, 0);
    const int64_t all = (int64_t)num_sms * (per > 0 ? per : 1);
    grid = (unsigned)(rows < all ? rows : all);
    return e;
}

template <typename T, int VPT, bool WARP, int MAXT>
cudaError_t launch_forward(const NormArgs& a, int threads, int num_sms, cudaStream_t st) {
    unsigned grid;
    const auto kern = norm_kernel<T, VPT, WARP, MAXT>;
    const int64_t units = WARP ? (a.R + threads / 32 - 1) / (threads / 32) : a.R;
    const cudaError_t e = resident(kern, threads, num_sms, units, grid);
    if (e != cudaSuccess) return e;
    return launch_k(kern, dim3(grid), dim3(threads), 0, st, false, a);
}

constexpr int kNormWarps = 4;  // warps of a CTA where warps are workers

template <typename T>
cudaError_t forward(const NormArgs& a, int num_sms, cudaStream_t st) {
    const int64_t nv = (a.d + Vec16<T>::kN - 1) / Vec16<T>::kN;
    if (nv <= 32) return launch_forward<T, 1, true, kNormWarps * 32>(a, kNormWarps * 32, num_sms, st);
    if (nv <= 512) return launch_forward<T, 1, false, 512>(a, cta_threads(nv, 1), num_sms, st);
    if (nv <= 1024) return launch_forward<T, 1, false, 1024>(a, cta_threads(nv, 1), num_sms, st);
    if (nv <= 2048) return launch_forward<T, 2, false, 1024>(a, cta_threads(nv, 2), num_sms, st);
    unsigned grid;
    const cudaError_t e = resident(norm_long_kernel<T>, 1024, num_sms, a.R, grid);
    if (e != cudaSuccess) return e;
    return launch_k(norm_long_kernel<T>, dim3(grid), dim3(1024), 0, st, false, a);
}

// how a row of d elements is held in the backward pass: by a warp, by a CTA (one or two vectors a thread), in passes
enum NormForm { BY_WARP, BY_CTA, BY_CTA_2, IN_PASSES };
NormForm backward_form(int d, fe_dtype dtype) {
    const int64_t v = dtype == FE_F32 ? 4 : 8, nv = (d + v - 1) / v;
    return nv <= 32 ? BY_WARP : nv <= 640 ? BY_CTA : nv <= 1024 ? BY_CTA_2 : IN_PASSES;
}

template <typename T>
cudaError_t backward(const NormArgs& a, fe_dtype dtype, cudaStream_t st) {
    const int64_t nv = (a.d + Vec16<T>::kN - 1) / Vec16<T>::kN;
    const int64_t workers = a.parts ? a.groups * a.parts : (a.groups + a.step - 1) / a.step;
    const dim3 grid((unsigned)workers);
    switch (backward_form(a.d, dtype)) {
        case BY_WARP:
            return launch_k(norm_backward_kernel<T, 1, true, kNormWarps * 32>, dim3((unsigned)((workers + kNormWarps - 1) / kNormWarps)),
                            dim3(kNormWarps * 32), 0, st, false, a, workers);
        case BY_CTA:
            return launch_k(norm_backward_kernel<T, 1, false, 640>, grid, dim3(cta_threads(nv, 1)), 0, st, false, a, workers);
        case BY_CTA_2:
            return launch_k(norm_backward_kernel<T, 2, false, 512>, grid, dim3(cta_threads(nv, 2)), 0, st, false, a, workers);
        default: return launch_k(norm_backward_long_kernel<T>, grid, dim3(1024), 0, st, false, a);
    }
}

}  // namespace

int64_t norm_backward_plan(NormArgs& a, fe_dtype dtype, int num_sms) {
    const int64_t v = dtype == FE_F32 ? 4 : 8, nv = (a.d + v - 1) / v;
    const NormForm form = backward_form(a.d, dtype);
    const int threads = form == BY_CTA_2 ? cta_threads(nv, 2) : cta_threads(nv, 1);
    // workers that fill the GPU once
    const int64_t want = form == BY_WARP ? (int64_t)num_sms * 16 : form == IN_PASSES ? num_sms : num_sms * (640 / threads > 0 ? 640 / threads : 1);
    const int64_t size = a.gate.p ? (a.gate_rows < a.R ? a.gate_rows : a.R) : a.R;
    a.gate_part = 1;
    a.groups = a.gate.p ? (a.R + a.gate_rows - 1) / a.gate_rows : 1;
    if (a.groups >= want) {
        a.gate_part = form == IN_PASSES;
        a.parts = 0;
        a.step = (a.groups + want - 1) / want;
        return (a.groups + a.step - 1) / a.step;
    }
    const int64_t parts = want / a.groups;
    a.parts = (int)(parts < size ? parts : size);
    a.step = 0;
    return a.groups * a.parts;
}

cudaError_t launch_block_norm(const NormArgs& a, fe_dtype dtype, int num_sms, cudaStream_t st) {
    return dtype == FE_F32 ? forward<float>(a, num_sms, st) : forward<bf16_t>(a, num_sms, st);
}

cudaError_t launch_block_norm_backward(const NormArgs& a, fe_dtype dtype, cudaStream_t st) {
    return dtype == FE_F32 ? backward<float>(a, dtype, st) : backward<bf16_t>(a, dtype, st);
}

}  // namespace fe
