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

// Rows on their way: a thread's vectors of the next rows, copied behind its back (cp.async) into slots that it
// alone writes and reads. NA arrays, DEPTH rows.
template <typename T, int NA, int VPT, int DEPTH>
struct RowRing {
    uint4* mine;  // [DEPTH][NA][VPT] vectors, `threads` apart
    int threads;
    __device__ __forceinline__ uint4* at(int slot, int array, int j) const { return mine + ((slot * NA + array) * VPT + j) * threads; }
    __device__ __forceinline__ void fetch(int slot, int array, const fe_mat& m, int64_t row, int c, int have, int j, bool vec) const {
        uint4* dst = at(slot, array, j);
        if (!m.p || have <= 0) return;
        const T* src = (const T*)m.p + row * m.row + c;
        if (vec && have >= Vec16<T>::kN) cp_async16(smem_u32(dst), src, true);
        else *dst = load_raw<T>(src, 0, have, false);
    }
};
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

constexpr int forward_depth(int vpt) { return vpt == 1 ? 4 : 3; }
constexpr int backward_depth(int vpt) { return vpt == 1 ? 3 : 2; }

template <typename T, int VPT, bool WARP, int MAXT, int CTAS>
__global__ void __launch_bounds__(MAXT, CTAS) norm_kernel(const __grid_constant__ NormArgs a) {
    constexpr int V = Vec16<T>::kN, D = forward_depth(VPT);
    extern __shared__ uint4 ring_mem[];
    __shared__ float buf[2][64];
    int turn = 0;
    const int nt = WARP ? 32 : blockDim.x, tid = WARP ? threadIdx.x % 32 : threadIdx.x;
    const int64_t step = WARP ? (int64_t)gridDim.x * (blockDim.x / 32) : gridDim.x;
    int64_t r = WARP ? (int64_t)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32 : blockIdx.x;
    const float inv_d = 1.f / (float)a.d;
    const RowRing<T, 2, VPT, D> ring{ring_mem + threadIdx.x, (int)blockDim.x};
    const auto fetch = [&](int64_t row, int slot) {
        if (row < a.R) {
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int c = (j * nt + tid) * V, have = a.d - c;
                ring.fetch(slot, 0, a.x, row, c, have, j, a.vec);
                ring.fetch(slot, 1, a.z, row, c, have, j, a.vec);
            }
        }
        cp_commit();
    };
    for (int i = 0; i < D - 1; ++i) fetch(r + i * step, i);
    int slot = 0;
    for (; r < a.R; r += step, slot = slot + 1 == D ? 0 : slot + 1) {
        cp_wait<D - 2>();
        float y[VPT][V], z[VPT][V];
        float scale_z = 1.f;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const bool has = (j * nt + tid) * V < a.d;
            Vec16<T>::widen(has ? *ring.at(slot, 0, j) : make_uint4(0, 0, 0, 0), y[j]);
            Vec16<T>::widen(has && a.z.p ? *ring.at(slot, 1, j) : make_uint4(0, 0, 0, 0), z[j]);
        }
        // (the slot that was read last: its row's outputs, which may be the inputs themselves, are rows before)
        fetch(r + (D - 1) * step, slot == 0 ? D - 1 : slot - 1);
        if (a.post) {
            float s[1] = {0.f};
#pragma unroll
            for (int j = 0; j < VPT; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) s[0] += z[j][i] * z[j][i];
            worker_sum<WARP, 1>(s, buf, turn);
            scale_z = rsqrtf(s[0] * inv_d + a.eps);
        }
        float s[1] = {0.f};
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = (j * nt + tid) * V, have = a.d - c;
            if (have > 0 && a.z.p) {
                float w[V];
                if (a.post) {
                    weights<T>(a.post_w, c, have, a.vec, a.offset, w);
#pragma unroll
                    for (int i = 0; i < V; ++i) z[j][i] *= scale_z * w[i];
                }
                if (a.gate.p) {
                    load_row<T, V>((const T*)a.gate.p + r / a.gate_rows * a.gate.row + c, have, a.vec, w);
#pragma unroll
                    for (int i = 0; i < V; ++i) z[j][i] *= w[i];
                }
#pragma unroll
                for (int i = 0; i < V; ++i) y[j][i] = fmaf(a.scale, z[j][i], y[j][i]);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += y[j][i] * y[j][i];
            if (a.y.p) store_row<T, V>((T*)a.y.p + r * a.y.row + c, have, a.vec, y[j]);
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
    cp_wait<0>();
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

// Pairs of neighbouring columns, and a thread's vector of them
template <typename T>
struct Pairs {
    static constexpr int N = Vec16<T>::kN / 2;
    uint64_t v[N];
    __device__ __forceinline__ void widen(const uint4& x) {
        if (sizeof(T) == 4) {
            v[0] = pair_f32(x.x, x.y);
            v[1] = pair_f32(x.z, x.w);
        } else {
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = pair_f32(w[i] << 16, w[i] & 0xFFFF0000u);
        }
    }
    __device__ __forceinline__ void floats(const float* f) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = pair_f32(__float_as_uint(f[2 * i]), __float_as_uint(f[2 * i + 1]));
    }
    __device__ __forceinline__ void to(float* f) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            f[2 * i] = low_f32(v[i]);
            f[2 * i + 1] = high_f32(v[i]);
        }
    }
};
__device__ __forceinline__ float pair_sum(uint64_t a) { return low_f32(a) + high_f32(a); }

// a thread's weights (w + offset; 1 without) or gates as they were loaded
template <typename T>
__device__ __forceinline__ void pair_weights(const uint4& raw, bool given, float offset, Pairs<T>& p) {
    p.widen(raw);
#pragma unroll
    for (int i = 0; i < Pairs<T>::N; ++i) p.v[i] = given ? add_x2(p.v[i], pair_f32(offset)) : pair_f32(1.f);
}

template <typename T, int VPT, bool WARP, int MAXT, int CTAS>
__global__ void __launch_bounds__(MAXT, CTAS) norm_backward_kernel(const __grid_constant__ NormArgs a, int64_t workers) {
    constexpr int V = Vec16<T>::kN, N = V / 2, D = backward_depth(VPT);
    extern __shared__ uint4 ring_mem[];
    __shared__ float buf[2][64];
    int turn = 0;
    const int nt = WARP ? 32 : blockDim.x, tid = WARP ? threadIdx.x % 32 : threadIdx.x;
    const int64_t worker = WARP ? (int64_t)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32 : blockIdx.x;
    if (worker >= workers) return;  // (a whole warp, where warps are workers)
    const float inv_d = 1.f / (float)a.d;
    int64_t r, r1;
    worker_rows(a, worker, r, r1);
    const RowRing<T, 4, VPT, D> ring{ring_mem + threadIdx.x, (int)blockDim.x};
    const auto fetch = [&](int64_t row, int slot) {
        if (row < r1) {
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int c = (j * nt + tid) * V, have = a.d - c;
                ring.fetch(slot, 0, a.x, row, c, have, j, a.vec);
                ring.fetch(slot, 1, a.z, row, c, have, j, a.vec);
                ring.fetch(slot, 2, a.dy, row, c, have, j, a.vec);
                ring.fetch(slot, 3, a.dn, row, c, have, j, a.vec);
            }
        }
        cp_commit();
    };
    uint64_t spre[VPT][N] = {}, spost[VPT][N] = {}, sgate[VPT][N] = {};
    int64_t group = 0, group_end = a.R;  // rows of the current gate
    if (a.gate.p) {
        group = r / a.gate_rows;
        group_end = (group + 1) * a.gate_rows;
    }
    // one vector a thread: weights and gates stay in registers; more: they are read again, from the first cache
    constexpr bool HOLD = VPT == 1;
    const int c0 = tid * V;
    uint4 hold_post = make_uint4(0, 0, 0, 0), hold_pre = hold_post, hold_gate = hold_post;
    const auto read_gate = [&] {
        if (HOLD && a.gate.p && c0 < a.d && r < r1) hold_gate = load_raw<T>(a.gate.p, group * a.gate.row + c0, a.d - c0, a.vec);
    };
    if (HOLD && c0 < a.d) {
        if (a.post_w) hold_post = load_raw<T>(a.post_w, c0, a.d - c0, a.vec);
        if (a.pre_w) hold_pre = load_raw<T>(a.pre_w, c0, a.d - c0, a.vec);
    }
    read_gate();
    const auto post_of = [&](int c, int have, Pairs<T>& w) {
        pair_weights<T>(HOLD || !a.post_w ? hold_post : load_raw<T>(a.post_w, c, have, a.vec), a.post_w, a.offset, w);
    };
    const auto pre_of = [&](int c, int have, Pairs<T>& w) {
        pair_weights<T>(HOLD || !a.pre_w ? hold_pre : load_raw<T>(a.pre_w, c, have, a.vec), a.pre_w, a.offset, w);
    };
    const auto gate_of = [&](int c, int have, Pairs<T>& w) {
        w.widen(HOLD ? hold_gate : load_raw<T>(a.gate.p, group * a.gate.row + c, have, a.vec));
    };
    for (int i = 0; i < D - 1; ++i) fetch(r + i, i);
    int slot = 0;
    for (; r < r1; ++r, slot = slot + 1 == D ? 0 : slot + 1) {
        cp_wait<D - 2>();
        float scale_z = 1.f;
        if (a.post) {
            float s[1] = {0.f};
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                if ((j * nt + tid) * V >= a.d) continue;
                Pairs<T> z;
                z.widen(*ring.at(slot, 1, j));
                uint64_t q = 0;
#pragma unroll
                for (int i = 0; i < N; ++i) q = fma_x2(z.v[i], z.v[i], q);
                s[0] += pair_sum(q);
            }
            worker_sum<WARP, 1>(s, buf, turn);
            scale_z = rsqrtf(s[0] * inv_d + a.eps);
        }
        // y, its square and (dn (w_pre + o)) y
        Pairs<T> y[VPT];
        float t[2] = {0.f, 0.f};
        const uint64_t sz = pair_f32(scale_z), sc = pair_f32(a.scale);
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = (j * nt + tid) * V, have = a.d - c;
            if (have <= 0) continue;
            Pairs<T> w;
            y[j].widen(*ring.at(slot, 0, j));
            if (a.z.p) {
                Pairs<T> p;
                p.widen(*ring.at(slot, 1, j));
                if (a.post) {
                    post_of(c, have, w);
#pragma unroll
                    for (int i = 0; i < N; ++i) p.v[i] = mul_x2(mul_x2(p.v[i], sz), w.v[i]);
                }
                if (a.gate.p) {
                    gate_of(c, have, w);
#pragma unroll
                    for (int i = 0; i < N; ++i) p.v[i] = mul_x2(p.v[i], w.v[i]);
                }
#pragma unroll
                for (int i = 0; i < N; ++i) y[j].v[i] = fma_x2(sc, p.v[i], y[j].v[i]);
            }
            if (a.dn.p) {
                Pairs<T> dn;
                dn.widen(*ring.at(slot, 3, j));
                pre_of(c, have, w);
                uint64_t q0 = 0, q1 = 0;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    q0 = fma_x2(y[j].v[i], y[j].v[i], q0);
                    q1 = fma_x2(mul_x2(dn.v[i], w.v[i]), y[j].v[i], q1);
                }
                t[0] += pair_sum(q0);
                t[1] += pair_sum(q1);
            }
        }
        float scale_y = 0.f, back = 0.f;
        if (a.dn.p) {
            worker_sum<WARP, 2>(t, buf, turn);
            scale_y = rsqrtf(t[0] * inv_d + a.eps);
            back = -t[1] * inv_d * scale_y * scale_y * scale_y;
        }
        const uint64_t sy = pair_f32(scale_y), by = pair_f32(back);
        float u[1] = {0.f};
        Pairs<T> b[VPT];  // dp (w_post + o)
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = (j * nt + tid) * V, have = a.d - c;
            if (have <= 0) continue;
            Pairs<T> w, dx;
            if (a.dy.p) {
                dx.widen(*ring.at(slot, 2, j));
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) dx.v[i] = 0;
            }
            if (a.dn.p) {
                Pairs<T> dn;
                dn.widen(*ring.at(slot, 3, j));
                pre_of(c, have, w);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const uint64_t ry = mul_x2(dn.v[i], sy);
                    spre[j][i] = fma_x2(ry, y[j].v[i], spre[j][i]);
                    dx.v[i] = fma_x2(by, y[j].v[i], fma_x2(ry, w.v[i], dx.v[i]));
                }
            }
            if (a.dx.p) {
                float f[V];
                dx.to(f);
                store_row<T, V>((T*)a.dx.p + r * a.dx.row + c, have, a.vec, f);
            }
            if (!a.z.p) continue;
            Pairs<T> z, g;
            z.widen(*ring.at(slot, 1, j));
            if (a.post) post_of(c, have, w);
            if (a.gate.p) gate_of(c, have, g);
            uint64_t q = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                uint64_t dp = mul_x2(dx.v[i], sc);
                const uint64_t zh = a.post ? mul_x2(z.v[i], sz) : z.v[i];
                if (a.gate.p) {
                    sgate[j][i] = fma_x2(dp, a.post ? mul_x2(zh, w.v[i]) : zh, sgate[j][i]);
                    dp = mul_x2(dp, g.v[i]);
                }
                if (a.post) {
                    spost[j][i] = fma_x2(dp, zh, spost[j][i]);
                    dp = mul_x2(dp, w.v[i]);
                    q = fma_x2(dp, z.v[i], q);
                }
                b[j].v[i] = dp;
            }
            u[0] += pair_sum(q);
        }
        if (a.post) worker_sum<WARP, 1>(u, buf, turn);
        if (a.dz.p) {
            const uint64_t bz = pair_f32(-u[0] * inv_d * scale_z * scale_z * scale_z);
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int c = (j * nt + tid) * V, have = a.d - c;
                if (have <= 0) continue;
                float f[V];
                if (a.post) {
                    Pairs<T> z;
                    z.widen(*ring.at(slot, 1, j));
#pragma unroll
                    for (int i = 0; i < N; ++i) b[j].v[i] = fma_x2(bz, z.v[i], mul_x2(sz, b[j].v[i]));
                }
                b[j].to(f);
                store_row<T, V>((T*)a.dz.p + r * a.dz.row + c, have, a.vec, f);
            }
        }
        fetch(r + D - 1, slot == 0 ? D - 1 : slot - 1);
        if (r + 1 == group_end || (r + 1 == r1 && !a.parts)) {  // the last row of a gate
            if (a.dgate.p && !a.part_gate) {
#pragma unroll
                for (int j = 0; j < VPT; ++j) {
                    const int c = (j * nt + tid) * V;
                    float f[V];
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        f[2 * i] = low_f32(sgate[j][i]);
                        f[2 * i + 1] = high_f32(sgate[j][i]);
                        sgate[j][i] = 0;
                    }
                    store_row<T, V>((T*)a.dgate.p + group * a.dgate.row + c, a.d - c, a.vec, f);
                }
            }
            if (a.gate.p) {
                ++group;
                group_end += a.gate_rows;
                if (r + 1 < r1) read_gate();
            }
        }
    }
    cp_wait<0>();
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int c = (j * nt + tid) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (c + i >= a.d) continue;
            const auto part = [&](const uint64_t* s) { return i & 1 ? high_f32(s[i / 2]) : low_f32(s[i / 2]); };
            if (a.part_pre) a.part_pre[worker * a.d + c + i] = part(spre[j]);
            if (a.part_post) a.part_post[worker * a.d + c + i] = part(spost[j]);
            if (a.part_gate) a.part_gate[worker * a.d + c + i] = part(sgate[j]);
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

constexpr int kNormWarps = 4;  // warps of a CTA where warps are workers

template <typename K>
cudaError_t resident(K kern, int threads, size_t smem, int num_sms, int64_t units, unsigned& grid) {
    int per = 0;
    const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kern, threads, smem);
    const int64_t all = (int64_t)num_sms * (per > 0 ? per : 1);
    grid = (unsigned)(units < all ? units : all);
    return e;
}

template <typename T, int VPT, bool WARP, int MAXT, int CTAS>
cudaError_t launch_forward(const NormArgs& a, int threads, int num_sms, cudaStream_t st) {
    unsigned grid;
    const auto kern = norm_kernel<T, VPT, WARP, MAXT, CTAS>;
    const size_t smem = (size_t)forward_depth(VPT) * 2 * VPT * threads * sizeof(uint4);
    const int64_t units = WARP ? (a.R + threads / 32 - 1) / (threads / 32) : a.R;
    const cudaError_t e = resident(kern, threads, smem, num_sms, units, grid);
    if (e != cudaSuccess) return e;
    return launch_k(kern, dim3(grid), dim3(threads), smem, st, false, a);
}

// vectors of a row: a warp's at most, a CTA's with one or two a thread, and more
constexpr int kWarpVecs = 32, kNarrow = 640, kOne = 1024, kTwo = 2048;

template <typename T>
cudaError_t forward(const NormArgs& a, int num_sms, cudaStream_t st) {
    const int64_t nv = (a.d + Vec16<T>::kN - 1) / Vec16<T>::kN;
    if (nv <= kWarpVecs) return launch_forward<T, 1, true, kNormWarps * 32, 8>(a, kNormWarps * 32, num_sms, st);
    if (nv <= kNarrow) return launch_forward<T, 1, false, kNarrow, 2>(a, cta_threads(nv, 1), num_sms, st);
    if (nv <= kOne) return launch_forward<T, 1, false, kOne, 1>(a, cta_threads(nv, 1), num_sms, st);
    if (nv <= kTwo) return launch_forward<T, 2, false, kOne, 1>(a, cta_threads(nv, 2), num_sms, st);
    unsigned grid;
    const cudaError_t e = resident(norm_long_kernel<T>, 1024, 0, num_sms, a.R, grid);
    if (e != cudaSuccess) return e;
    return launch_k(norm_long_kernel<T>, dim3(grid), dim3(1024), 0, st, false, a);
}

// how a row of d elements is held in the backward pass: by a warp, by a CTA (one or two vectors a thread), in passes
enum NormForm { BY_WARP, BY_CTA, BY_CTA_2, IN_PASSES };
NormForm backward_form(int64_t nv) { return nv <= kWarpVecs ? BY_WARP : nv <= kNarrow ? BY_CTA : nv <= kOne ? BY_CTA_2 : IN_PASSES; }
int form_threads(NormForm f, int64_t nv) {
    return f == BY_WARP ? kNormWarps * 32 : f == IN_PASSES ? 1024 : cta_threads(nv, f == BY_CTA ? 1 : 2);
}
int64_t row_vecs(int d, fe_dtype dtype) { return dtype == FE_F32 ? ((int64_t)d + 3) / 4 : ((int64_t)d + 7) / 8; }

template <typename T>
cudaError_t backward(const NormArgs& a, fe_dtype dtype, cudaStream_t st) {
    const int64_t nv = row_vecs(a.d, dtype);
    const NormForm form = backward_form(nv);
    const int threads = form_threads(form, nv);
    const int64_t workers = a.parts ? a.groups * a.parts : (a.groups + a.step - 1) / a.step;
    const int vpt = form == BY_CTA_2 ? 2 : 1;
    const size_t smem = (size_t)backward_depth(vpt) * 4 * vpt * threads * sizeof(uint4);
    const dim3 grid((unsigned)workers);
    switch (form) {
        case BY_WARP:
            return launch_k(norm_backward_kernel<T, 1, true, kNormWarps * 32, 4>, dim3((unsigned)((workers + kNormWarps - 1) / kNormWarps)),
                            dim3(threads), smem, st, false, a, workers);
        case BY_CTA:
            if (threads <= 320) return launch_k(norm_backward_kernel<T, 1, false, 320, 2>, grid, dim3(threads), smem, st, false, a, workers);
            return launch_k(norm_backward_kernel<T, 1, false, kNarrow, 1>, grid, dim3(threads), smem, st, false, a, workers);
        case BY_CTA_2:
            return launch_k(norm_backward_kernel<T, 2, false, 512, 1>, grid, dim3(threads), smem, st, false, a, workers);
        default: return launch_k(norm_backward_long_kernel<T>, grid, dim3(threads), 0, st, false, a);
    }
}

template <typename K>
cudaError_t allow(K kern, size_t bytes) {
    return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <typename T>
cudaError_t prepare() {
    cudaError_t e;
    const size_t f = forward_depth(1) * 2 * sizeof(uint4), f2 = forward_depth(2) * 4 * sizeof(uint4), b = backward_depth(1) * 4 * sizeof(uint4);
    if ((e = allow(norm_kernel<T, 1, false, kNarrow, 2>, f * kNarrow)) != cudaSuccess) return e;
    if ((e = allow(norm_kernel<T, 1, false, kOne, 1>, f * kOne)) != cudaSuccess) return e;
    if ((e = allow(norm_kernel<T, 2, false, kOne, 1>, f2 * kOne)) != cudaSuccess) return e;
    if ((e = allow(norm_backward_kernel<T, 1, false, 320, 2>, b * 320)) != cudaSuccess) return e;
    if ((e = allow(norm_backward_kernel<T, 1, false, kNarrow, 1>, b * kNarrow)) != cudaSuccess) return e;
    return allow(norm_backward_kernel<T, 2, false, 512, 1>, backward_depth(2) * 8 * sizeof(uint4) * 512);
}

}  // namespace

cudaError_t norm_prepare() {
    const cudaError_t e = prepare<float>();
    return e != cudaSuccess ? e : prepare<bf16_t>();
}

int64_t norm_backward_plan(NormArgs& a, fe_dtype dtype, int num_sms) {
    const int64_t nv = row_vecs(a.d, dtype);
    const NormForm form = backward_form(nv);
    // workers that fill the GPU once: 16 warps an SM, or the CTAs of some 640 threads
    const int ctas = 640 / form_threads(form, nv);
    const int64_t want = (int64_t)num_sms * (form == BY_WARP ? 16 : ctas > 0 ? ctas : 1);
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
