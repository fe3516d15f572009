// The norms behind a block and before the next with the block's gate and residual (fe_block_norm),
// and their gradient. Bound by memory traffic: a row's vectors are read once, stay in registers for
// the statistics that depend on one another, and are written once.
//
//   forward   p = z rz (w_post + o), y = x + s g p, n = y ry (w_pre + o), r = 1 / sqrt(mean of squares + eps)
//   backward  with a = dn (w_pre + o):
//             dx = dy + ry a - y ry^3 mean(a y),  dw_pre = sum dn y ry
//             with b = dx s g (w_post + o):  dz = rz b - z rz^3 mean(b z)
//             with t = sum dx z rz over the rows of a gate:  dg = s (w_post + o) t,  dw_post = sum s g t
//             (y is computed again from x and z, so nothing rounded stands in for it)
//
// Measured (GB300, 16379 rows of 5120 bfloat16, gate, both norms): forward 105 us (6.4 TB/s; with one vector a thread
// 134, loads in registers ahead instead of copies 143 to 193), gradient 174 us over 148 us of bytes, bound by
// the latency of shared memory and by issue (57 % of the slots; with CTAs of 640 threads 325; separate sums for
// gate and weight 30 % more registers and work; with the ring's stride in a register, not a constant of the
// kernel, 223).
//
// A worker is a CTA, or a warp where a row is at most 64 vectors of 16 bytes; its threads own
// columns, so that the sums over rows stay in registers. The next row's loads are in flight while
// a row's statistics are reduced.
#include <atomic>

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

// a thread's vector of a row; FULL: rows are whole vectors on their boundaries
template <typename T, bool FULL>
__device__ __forceinline__ uint4 load_vec(const T* p, int have, bool vec) {
    if (FULL) return *reinterpret_cast<const uint4*>(p);
    return load_raw<T>(p, 0, have, vec);
}
template <typename T, bool FULL>
__device__ __forceinline__ void store_vec(T* p, int have, bool vec, const float* f) {
    if (FULL) *reinterpret_cast<uint4*>(p) = pack16<T>(f);
    else store_row<T, Vec16<T>::kN>(p, have, vec, f);
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

// Rows on their way: a thread's vectors of the next rows, copied behind its back (cp.async) into slots that it
// alone writes and reads. NA arrays, DEPTH rows.
template <typename T, int NA, int VPT, bool FULL, int S>
struct RowRing {
    uint4* mine;  // [DEPTH][NA][VPT] vectors, S apart
    __device__ __forceinline__ uint4* at(int slot, int array, int j) const { return mine + ((slot * NA + array) * VPT + j) * S; }
    __device__ __forceinline__ void fetch(int slot, int array, int j, const T* src, int have, bool vec) const {
        uint4* dst = at(slot, array, j);
        if (FULL || (vec && have >= Vec16<T>::kN)) cp_async16(smem_u32(dst), src, true);
        else *dst = load_raw<T>(src, 0, have, false);
    }
};
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

constexpr int kNormDepth = 2;  // rows of a worker on their way
constexpr int back_depth(int room) { return room <= 512 ? kNormDepth : 1; }  // in the backward pass: what 227 KB hold

// the group of rows that share a gate (rows are below 2^30)
__device__ __forceinline__ int64_t group_of(const NormArgs& a, int64_t r) {
    return a.gate_rows >= a.R ? 0 : (uint32_t)r / (uint32_t)a.gate_rows;
}

// What a kernel may take for granted: nothing; rows that are whole vectors on their boundaries; and with them every
// operand but the gate and, in the backward pass, w_post, which are read outside its loop over the rows
// (16379 x 5120 bfloat16 with a gate: gradient 174 us, 198 with the questions asked in the loop, forward 105, 112).
enum Given { ANY, WHOLE, ALL_GIVEN };
template <typename T, int VPT, bool WARP, int MAXT, int CTAS, int KIND>
__global__ void __launch_bounds__(MAXT, CTAS) norm_kernel(const __grid_constant__ NormArgs a) {
    constexpr int V = Vec16<T>::kN, N = V / 2, D = kNormDepth;
    constexpr bool FULL = KIND >= WHOLE, ALL = KIND == ALL_GIVEN;
    const bool has_z = ALL || a.z.p, has_post = ALL || a.post;
    extern __shared__ uint4 ring_mem[];
    __shared__ float buf[2][64];
    int turn = 0;
    const int nt = WARP ? 32 : blockDim.x, tid = WARP ? threadIdx.x % 32 : threadIdx.x;
    const int64_t step = WARP ? (int64_t)gridDim.x * (blockDim.x / 32) : gridDim.x;
    int64_t r = WARP ? (int64_t)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32 : blockIdx.x;
    const float inv_d = 1.f / (float)a.d;
    const RowRing<T, 2, VPT, FULL, MAXT> ring{ring_mem + threadIdx.x};
    const T *px = (const T*)a.x.p + r * a.x.row, *pz = (const T*)a.z.p + r * a.z.row;  // the next row to fetch
    const int64_t sx = step * a.x.row, sz_ = step * a.z.row;
    int64_t next = r;
    const auto fetch = [&](int slot) {
        if (next < a.R) {
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int c = (j * nt + tid) * V, have = a.d - c;
                if (have <= 0) continue;
                ring.fetch(slot, 0, j, px + c, have, a.vec);
                if (has_z) ring.fetch(slot, 1, j, pz + c, have, a.vec);
            }
        }
        cp_commit();
        px += sx;
        pz += sz_;
        next += step;
    };
    // a thread's weights as they are stored, behind the rows
    const auto hold = [&](int array, int j) { return ring_mem + threadIdx.x + ((D * 2 + array) * VPT + j) * MAXT; };
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int c = (j * nt + tid) * V, have = a.d - c;
        if (a.post_w && have > 0) *hold(0, j) = load_vec<T, FULL>((const T*)a.post_w + c, have, a.vec);
        if (a.pre_w && have > 0) *hold(1, j) = load_vec<T, FULL>((const T*)a.pre_w + c, have, a.vec);
    }
    const auto held = [&](const void* w, int array, int j, Pairs<T>& p) {
        if (!ALL && !w) {
#pragma unroll
            for (int i = 0; i < N; ++i) p.v[i] = pair_f32(1.f);
            return;
        }
        p.widen(*hold(array, j));
#pragma unroll
        for (int i = 0; i < N; ++i) p.v[i] = add_x2(p.v[i], pair_f32(a.offset));
    };
    T *py = (T*)a.y.p + r * a.y.row, *pn = (T*)a.n.p + r * a.n.row;
    const uint64_t sc = pair_f32(a.scale);
    for (int i = 0; i < D; ++i) fetch(i);
    int slot = 0;
    for (; r < a.R; r += step, slot = slot + 1 == D ? 0 : slot + 1) {
        cp_wait<D - 1>();
        Pairs<T> y[VPT], z[VPT];
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const bool has = (j * nt + tid) * V < a.d;
            y[j].widen(has ? *ring.at(slot, 0, j) : make_uint4(0, 0, 0, 0));
            z[j].widen(has && has_z ? *ring.at(slot, 1, j) : make_uint4(0, 0, 0, 0));
        }
        fetch(slot);  // (outputs may be the inputs themselves: rows that have been read)
        float scale_z = 1.f;
        if (has_post) {
            uint64_t q = 0;
#pragma unroll
            for (int j = 0; j < VPT; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) q = fma_x2(z[j].v[i], z[j].v[i], q);
            float s[1] = {pair_sum(q)};
            worker_sum<WARP, 1>(s, buf, turn);
            scale_z = rsqrtf(s[0] * inv_d + a.eps);
        }
        uint64_t q = 0;
        const T* gate = (const T*)a.gate.p + (a.gate.p ? group_of(a, r) * a.gate.row : 0);
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = (j * nt + tid) * V, have = a.d - c;
            if (have <= 0) continue;
            if (has_z) {
                Pairs<T> w;
                if (has_post) {
                    held(a.post_w, 0, j, w);
                    const uint64_t sz = pair_f32(scale_z);
#pragma unroll
                    for (int i = 0; i < N; ++i) z[j].v[i] = mul_x2(mul_x2(z[j].v[i], sz), w.v[i]);
                }
                if (a.gate.p) {
                    w.widen(load_vec<T, FULL>(gate + c, have, a.vec));
#pragma unroll
                    for (int i = 0; i < N; ++i) z[j].v[i] = mul_x2(z[j].v[i], w.v[i]);
                }
#pragma unroll
                for (int i = 0; i < N; ++i) y[j].v[i] = fma_x2(sc, z[j].v[i], y[j].v[i]);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) q = fma_x2(y[j].v[i], y[j].v[i], q);
            if (ALL || a.y.p) {
                float f[V];
                y[j].to(f);
                store_vec<T, FULL>(py + c, have, a.vec, f);
            }
        }
        py += step * a.y.row;
        if (!ALL && !a.n.p) continue;
        float s[1] = {pair_sum(q)};
        worker_sum<WARP, 1>(s, buf, turn);
        const uint64_t sy = pair_f32(rsqrtf(s[0] * inv_d + a.eps));
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = (j * nt + tid) * V, have = a.d - c;
            if (have <= 0) continue;
            Pairs<T> w;
            held(a.pre_w, 1, j, w);
#pragma unroll
            for (int i = 0; i < N; ++i) w.v[i] = mul_x2(mul_x2(y[j].v[i], sy), w.v[i]);
            float f[V];
            w.to(f);
            store_vec<T, FULL>(pn + c, have, a.vec, f);
        }
        pn += step * a.n.row;
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

// Half a vector: two pairs of bfloat16 columns, or one of float32. The backward pass works through halves, so
// that little more than the sums over rows and a row's y is in registers at any time.
template <typename T>
struct Half {
    static constexpr int N = Vec16<T>::kN / 4;
    uint64_t v[N];
    __device__ __forceinline__ void widen(const uint4* p, int h) {
        const uint2 x = reinterpret_cast<const uint2*>(p)[h];
        if (sizeof(T) == 4) {
            v[0] = pair_f32(x.x, x.y);
        } else {
            v[0] = pair_f32(x.x << 16, x.x & 0xFFFF0000u);
            v[N - 1] = pair_f32(x.y << 16, x.y & 0xFFFF0000u);
        }
    }
    __device__ __forceinline__ uint2 pack() const {
        if (sizeof(T) == 4) return make_uint2((uint32_t)v[0], (uint32_t)(v[0] >> 32));
        return make_uint2(pack_bf16(low_f32(v[0]), high_f32(v[0])), pack_bf16(low_f32(v[N - 1]), high_f32(v[N - 1])));
    }
};
// a thread's weights as held: w + offset, or 1
template <typename T>
__device__ __forceinline__ void half_weights(const uint4* held, int h, bool given, uint64_t offset, Half<T>& p) {
    if (given) {
        p.widen(held, h);
#pragma unroll
        for (int i = 0; i < Half<T>::N; ++i) p.v[i] = add_x2(p.v[i], offset);
    } else {
#pragma unroll
        for (int i = 0; i < Half<T>::N; ++i) p.v[i] = pair_f32(1.f);
    }
}
template <typename T, bool FULL>
__device__ __forceinline__ void store_packed(T* p, int have, bool vec, const uint2& lo, const uint2& hi) {
    const uint4 x = make_uint4(lo.x, lo.y, hi.x, hi.y);
    if (FULL || (vec && have >= Vec16<T>::kN)) {
        *reinterpret_cast<uint4*>(p) = x;
    } else {
        const T* e = reinterpret_cast<const T*>(&x);
#pragma unroll
        for (int i = 0; i < Vec16<T>::kN; ++i)
            if (i < have) p[i] = e[i];
    }
}
template <typename T, int VPT, bool WARP, int MAXT, int CTAS, int KIND>
__global__ void __launch_bounds__(MAXT, CTAS) norm_backward_kernel(const __grid_constant__ NormArgs a, int64_t workers) {
    constexpr int V = Vec16<T>::kN, N = V / 2, HN = N / 2, D = back_depth(MAXT);
    constexpr bool FULL = KIND >= WHOLE, ALL = KIND == ALL_GIVEN;
    const bool has_z = ALL || a.z.p, has_dy = ALL || a.dy.p, has_dn = ALL || a.dn.p, has_post = ALL || a.post;
    extern __shared__ uint4 ring_mem[];
    __shared__ float buf[2][64];
    int turn = 0;
    const int nt = WARP ? 32 : blockDim.x, tid = WARP ? threadIdx.x % 32 : threadIdx.x;
    const int64_t worker = WARP ? (int64_t)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32 : blockIdx.x;
    if (worker >= workers) return;  // (a whole warp, where warps are workers)
    const float inv_d = 1.f / (float)a.d;
    int64_t r, r1;
    worker_rows(a, worker, r, r1);
    // The half of a vector that a thread takes first: lanes 8 to 15 of every 16 the upper one, so that the 8-byte
    // reads of 16 lanes, 16 bytes apart, meet every bank once. y, sdx and spre are in a thread's own order. (float32 rows
    // of 5120 184 us, 206 without; bfloat16 in order: the selections cost more than the banks, 150 us against 156.)
    const int flip = sizeof(T) == 4 ? threadIdx.x >> 3 & 1 : 0;
    const RowRing<T, 4, VPT, FULL, MAXT> ring{ring_mem + threadIdx.x};
    const auto fetch = [&](int64_t row, int slot) {
        if (row < r1) {
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int c = (j * nt + tid) * V, have = a.d - c;
                if (have <= 0) continue;
                ring.fetch(slot, 0, j, (const T*)a.x.p + row * a.x.row + c, have, a.vec);
                if (has_z) ring.fetch(slot, 1, j, (const T*)a.z.p + row * a.z.row + c, have, a.vec);
                if (has_dy) ring.fetch(slot, 2, j, (const T*)a.dy.p + row * a.dy.row + c, have, a.vec);
                if (has_dn) ring.fetch(slot, 3, j, (const T*)a.dn.p + row * a.dn.row + c, have, a.vec);
            }
        }
        cp_commit();
    };
    uint64_t spre[VPT][N] = {}, sdx[VPT][N] = {};  // sums of dn y ry, and over a gate's rows of dx zh
    int64_t group = 0, group_end = a.R;  // rows of the current gate
    if (a.gate.p) {
        group = group_of(a, r);
        group_end = (group + 1) * a.gate_rows;
    }
    // a thread's w_pre as it is stored, and s g (w_post + o) of the current gate in float32, behind the rows
    const auto hold = [&](int array, int j) { return ring_mem + threadIdx.x + ((D * 4 + array) * VPT + j) * MAXT; };
    const auto factor = [&](int j, int h) { return reinterpret_cast<uint64_t*>(hold(sizeof(T) == 2 ? 1 + h : 1, j)) + (sizeof(T) == 2 ? 0 : h); };
    // gates and post weights of a vector's columns, and what they are multiplied with
    const auto gates_of = [&](int j, float* g, float* w) {
        const int c = (j * nt + tid) * V, have = a.d - c;
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = a.scale;
        if (a.gate.p) {
            load_row<T, V>((const T*)a.gate.p + group * a.gate.row + c, have, a.vec, g);
#pragma unroll
            for (int i = 0; i < V; ++i) g[i] *= a.scale;
        }
        weights<T>(a.post_w, c, have, a.vec, a.offset, w);
    };
    const auto read_gate = [&] {
        if (!has_z || r >= r1) return;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            if ((j * nt + tid) * V >= a.d) continue;
            float g[V], w[V];
            gates_of(j, g, w);
#pragma unroll
            for (int i = 0; i < N; ++i)
                factor(j, i / HN)[i % HN] = pair_f32(__float_as_uint(g[2 * i] * w[2 * i]), __float_as_uint(g[2 * i + 1] * w[2 * i + 1]));
        }
    };
    // At the end of a gate's rows: dgate = s (w_post + o) sum dx zh, dw_post += s g sum dx zh. A worker of several
    // gates adds dw_post up in its own part of memory.
    bool begun = false;
    const auto end_gate = [&] {
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = (j * nt + tid) * V, have = a.d - c;
            if (have <= 0) continue;
            float g[V], w[V], t[V];
            gates_of(j, g, w);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint64_t v = flip ? sdx[j][i ^ HN] : sdx[j][i];
                t[2 * i] = low_f32(v);
                t[2 * i + 1] = high_f32(v);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) sdx[j][i] = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                g[i] *= t[i];
                w[i] *= a.scale * t[i];
            }
            if (a.part_gate) store_row<float, V>(a.part_gate + worker * a.d + c, have, false, w);
            else if (a.dgate.p) store_row<T, V>((T*)a.dgate.p + group * a.dgate.row + c, have, a.vec, w);
            if (a.part_post) {
                float* p = a.part_post + worker * a.d + c;
                if (begun) {
                    load_row<float, V>(p, have, false, t);
#pragma unroll
                    for (int i = 0; i < V; ++i) g[i] += t[i];
                }
                store_row<float, V>(p, have, false, g);
            }
        }
        begun = true;
    };
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int c = (j * nt + tid) * V;
        if (a.pre_w && c < a.d) *hold(0, j) = load_vec<T, FULL>((const T*)a.pre_w + c, a.d - c, a.vec);
    }
    read_gate();
    if (r >= r1) {  // (more workers than rows in a short last group)
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = (j * nt + tid) * V;
            for (int i = 0; i < V && c + i < a.d; ++i) {
                if (a.part_gate) a.part_gate[worker * a.d + c + i] = 0.f;
                if (a.part_post) a.part_post[worker * a.d + c + i] = 0.f;
            }
        }
    }
    const auto pre_of = [&](int j, int h, Half<T>& w) { half_weights<T>(hold(0, j), h ^ flip, ALL || a.pre_w, pair_f32(a.offset), w); };
    for (int i = 0; i < D; ++i) fetch(r + i, i);
    int slot = 0;
    for (; r < r1; ++r, slot = slot + 1 == D ? 0 : slot + 1) {
        cp_wait<D - 1>();
        float scale_z = 1.f;
        if (has_post) {
            uint64_t q = 0;
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                if ((j * nt + tid) * V >= a.d) continue;
                Pairs<T> z;
                z.widen(*ring.at(slot, 1, j));
#pragma unroll
                for (int i = 0; i < N; ++i) q = fma_x2(z.v[i], z.v[i], q);
            }
            float s[1] = {pair_sum(q)};
            worker_sum<WARP, 1>(s, buf, turn);
            scale_z = rsqrtf(s[0] * inv_d + a.eps);
        }
        // y, its square and (dn (w_pre + o)) y
        uint64_t y[VPT][N], q0 = 0, q1 = 0;
        const uint64_t sz = pair_f32(scale_z);
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            if ((j * nt + tid) * V >= a.d) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                Half<T> f, w;
                f.widen(ring.at(slot, 0, j), h ^ flip);
                if (has_z) {
                    Half<T> p;
                    p.widen(ring.at(slot, 1, j), h ^ flip);
#pragma unroll
                    for (int i = 0; i < HN; ++i) f.v[i] = fma_x2(mul_x2(p.v[i], sz), factor(j, h ^ flip)[i], f.v[i]);
                }
                if (has_dn) {
                    Half<T> dn;
                    dn.widen(ring.at(slot, 3, j), h ^ flip);
                    pre_of(j, h, w);
#pragma unroll
                    for (int i = 0; i < HN; ++i) {
                        q0 = fma_x2(f.v[i], f.v[i], q0);
                        q1 = fma_x2(mul_x2(dn.v[i], w.v[i]), f.v[i], q1);
                    }
                }
#pragma unroll
                for (int i = 0; i < HN; ++i) y[j][h * HN + i] = f.v[i];
            }
        }
        float scale_y = 0.f, back = 0.f;
        if (has_dn) {
            float t[2] = {pair_sum(q0), pair_sum(q1)};
            worker_sum<WARP, 2>(t, buf, turn);
            scale_y = rsqrtf(t[0] * inv_d + a.eps);
            back = -t[1] * inv_d * scale_y * scale_y * scale_y;
        }
        const uint64_t sy = pair_f32(scale_y), by = pair_f32(back);
        uint64_t q = 0;
        // y becomes dx s g (w_post + o)
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = (j * nt + tid) * V, have = a.d - c;
            if (have <= 0) continue;
            uint2 out[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                Half<T> w, dx;
                if (has_dy) {
                    dx.widen(ring.at(slot, 2, j), h ^ flip);
                } else {
#pragma unroll
                    for (int i = 0; i < HN; ++i) dx.v[i] = 0;
                }
                if (has_dn) {
                    Half<T> dn;
                    dn.widen(ring.at(slot, 3, j), h ^ flip);
                    pre_of(j, h, w);
#pragma unroll
                    for (int i = 0; i < HN; ++i) {
                        const int k = h * HN + i;
                        const uint64_t ry = mul_x2(dn.v[i], sy);
                        spre[j][k] = fma_x2(ry, y[j][k], spre[j][k]);
                        dx.v[i] = fma_x2(by, y[j][k], fma_x2(ry, w.v[i], dx.v[i]));
                    }
                }
                out[h] = dx.pack();
                if (has_z) {
                    Half<T> z;
                    z.widen(ring.at(slot, 1, j), h ^ flip);
#pragma unroll
                    for (int i = 0; i < HN; ++i) {
                        const int k = h * HN + i;
                        const uint64_t dp = mul_x2(dx.v[i], factor(j, h ^ flip)[i]);
                        sdx[j][k] = fma_x2(dx.v[i], mul_x2(z.v[i], sz), sdx[j][k]);
                        q = fma_x2(dp, z.v[i], q);
                        y[j][k] = dp;
                    }
                }
            }
            if (ALL || a.dx.p) store_packed<T, FULL>((T*)a.dx.p + r * a.dx.row + c, have, a.vec, flip ? out[1] : out[0], flip ? out[0] : out[1]);
        }
        float u[1] = {pair_sum(q)};
        if (has_post) worker_sum<WARP, 1>(u, buf, turn);
        if (ALL || a.dz.p) {
            const uint64_t bz = pair_f32(-u[0] * inv_d * scale_z * scale_z * scale_z);
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int c = (j * nt + tid) * V, have = a.d - c;
                if (have <= 0) continue;
                uint2 out[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    Half<T> z, dz;
                    z.widen(ring.at(slot, 1, j), h ^ flip);
#pragma unroll
                    for (int i = 0; i < HN; ++i) {
                        const uint64_t b = y[j][h * HN + i];
                        dz.v[i] = has_post ? fma_x2(bz, z.v[i], mul_x2(sz, b)) : b;
                    }
                    out[h] = dz.pack();
                }
                store_packed<T, FULL>((T*)a.dz.p + r * a.dz.row + c, have, a.vec, flip ? out[1] : out[0], flip ? out[0] : out[1]);
            }
        }
        fetch(r + D, slot);
        if (r + 1 == group_end || r + 1 == r1) {  // the last of a gate's rows here
            end_gate();
            if (a.gate.p && r + 1 < r1) {
                ++group;
                group_end += a.gate_rows;
                read_gate();
            }
        }
    }
    cp_wait<0>();
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int c = (j * nt + tid) * V;
        if (!a.part_pre || c >= a.d) continue;
        float f[V];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint64_t v = flip ? spre[j][i ^ HN] : spre[j][i];
            f[2 * i] = low_f32(v);
            f[2 * i + 1] = high_f32(v);
        }
        store_row<float, V>(a.part_pre + worker * a.d + c, a.d - c, false, f);
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

// A grid of the CTAs that fit at once, no more than `units`. How many fit an SM is asked once for each kernel and
// size of a CTA (`known`, by warps).
using Known = std::atomic<int>[33];
template <typename K>
cudaError_t resident(K kern, Known& known, int threads, size_t smem, int num_sms, int64_t units, unsigned& grid) {
    int per = known[threads / 32].load(std::memory_order_relaxed);
    if (!per) {
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kern, threads, smem);
        if (e != cudaSuccess) return e;
        if (per < 1) per = 1;
        known[threads / 32].store(per, std::memory_order_relaxed);
    }
    const int64_t all = (int64_t)num_sms * per;
    grid = (unsigned)(units < all ? units : all);
    return cudaSuccess;
}

// rows that are whole vectors on 16-byte boundaries
template <typename T> bool whole(const NormArgs& a) { return a.vec && a.d % Vec16<T>::kN == 0; }

template <typename T, int VPT, bool WARP, int MAXT, int CTAS>
cudaError_t launch_forward(const NormArgs& a, int threads, int num_sms, cudaStream_t st) {
    unsigned grid;
    const bool all = a.z.p && a.post && a.post_w && a.pre_w && a.y.p && a.n.p;
    const int kind = !whole<T>(a) ? ANY : all ? ALL_GIVEN : WHOLE;
    const auto kern = kind == ANY     ? norm_kernel<T, VPT, WARP, MAXT, CTAS, ANY>
                      : kind == WHOLE ? norm_kernel<T, VPT, WARP, MAXT, CTAS, WHOLE>
                                      : norm_kernel<T, VPT, WARP, MAXT, CTAS, ALL_GIVEN>;
    const size_t smem = (size_t)(kNormDepth + 1) * 2 * VPT * MAXT * sizeof(uint4);
    const int64_t units = WARP ? (a.R + threads / 32 - 1) / (threads / 32) : a.R;
    static Known known[3];
    const cudaError_t e = resident(kern, known[kind], threads, smem, num_sms, units, grid);
    if (e != cudaSuccess) return e;
    return launch_k(kern, dim3(grid), dim3(threads), smem, st, false, a);
}

// vectors of a row: a warp's at most, a CTA's with one or two a thread, and more
constexpr int kWarpVecs = 32, kOne = 1024, kTwo = 2048;

template <typename T>
cudaError_t forward(const NormArgs& a, int num_sms, cudaStream_t st) {
    const int64_t nv = (a.d + Vec16<T>::kN - 1) / Vec16<T>::kN;
    if (nv <= kWarpVecs) return launch_forward<T, 1, true, kNormWarps * 32, 8>(a, kNormWarps * 32, num_sms, st);
    if (nv <= 2 * kWarpVecs) return launch_forward<T, 2, true, kNormWarps * 32, 8>(a, kNormWarps * 32, num_sms, st);
    if (nv <= 128) return launch_forward<T, 1, false, 128, 8>(a, cta_threads(nv, 1), num_sms, st);
    if (nv <= 256) return launch_forward<T, 1, false, 256, 4>(a, cta_threads(nv, 1), num_sms, st);
    if (nv <= 384) return launch_forward<T, 2, false, 192, 5>(a, cta_threads(nv, 2), num_sms, st);
    if (nv <= 640) return launch_forward<T, 2, false, 320, 3>(a, cta_threads(nv, 2), num_sms, st);
    if (nv <= kOne) return launch_forward<T, 2, false, 512, 2>(a, cta_threads(nv, 2), num_sms, st);
    if (nv <= kTwo) return launch_forward<T, 2, false, kOne, 1>(a, cta_threads(nv, 2), num_sms, st);
    unsigned grid;
    static Known known;
    const cudaError_t e = resident(norm_long_kernel<T>, known, 1024, 0, num_sms, a.R, grid);
    if (e != cudaSuccess) return e;
    return launch_k(norm_long_kernel<T>, dim3(grid), dim3(1024), 0, st, false, a);
}

// how a row of d elements is held in the backward pass: by a warp (one or two vectors a lane), by a CTA, in passes
enum NormForm { BY_WARP, BY_WARP_2, BY_CTA, IN_PASSES };
NormForm backward_form(int64_t nv) { return nv <= kWarpVecs ? BY_WARP : nv <= 2 * kWarpVecs ? BY_WARP_2 : nv <= kTwo ? BY_CTA : IN_PASSES; }
int form_threads(NormForm f, int64_t nv) {
    return f <= BY_WARP_2 ? kNormWarps * 32 : f == IN_PASSES ? 1024 : cta_threads(nv, 2);
}
// The kernels of the backward pass that hold a row: vectors a thread, threads at most (and room for them in the
// ring), whether warps are workers, and the CTAs of an SM that registers are kept for. Two vectors a thread wherever
// a row has enough: half the reductions' work for each element (128 MB of x, gradient without a gate: rows of 1024
// float32 143 us, with one vector 192; 2048 bfloat16 161, 221; 2560 bfloat16 170, 205), and a warp with two vectors
// a lane before a CTA of 64 threads (rows of 320 bfloat16 214 us, 240; 512 alike). Long rows keep one row on its way
// and still beat passes over memory (5120 float32 211 us, 557; 8192 float32 190, 421).
struct BackKernel {
    int vpt, room;
    bool warp;
    int ctas;
    int ctas_f32 = ctas;  // (a third CTA of 192 threads: float32 rows of 1536 149 us, 165 without; bfloat16 of 2880 214, 202)
};
constexpr BackKernel kBack[] = {{1, kNormWarps * 32, true, 5}, {2, kNormWarps * 32, true, 5}, {2, 64, false, 9},
                                {2, 128, false, 5},            {2, 160, false, 4},            {2, 192, false, 2, 3},
                                {2, 320, false, 2},            {2, 512, false, 1},            {2, 768, false, 1},
                                {2, 1024, false, 1}};
constexpr int kBacks = sizeof(kBack) / sizeof(kBack[0]);
constexpr size_t back_smem(int i) { return (size_t)(back_depth(kBack[i].room) * 4 + 3) * kBack[i].vpt * kBack[i].room * sizeof(uint4); }
int back_kernel(NormForm f, int threads) {
    if (f <= BY_WARP_2) return f;
    int i = 2;
    while (kBack[i].room < threads) ++i;
    return i;
}
// CTAs of each that fit an SM, as the device says when a handle's first gradient is prepared
std::atomic<int> back_fit[2][kBacks];
int64_t row_vecs(int d, fe_dtype dtype) { return dtype == FE_F32 ? ((int64_t)d + 3) / 4 : ((int64_t)d + 7) / 8; }

// f(i, what it takes for granted, kernel) for every kernel of the backward pass
template <typename T, int I, typename F>
void each_back(const F& f) {
    if constexpr (I < kBacks) {
        constexpr BackKernel k = kBack[I];
        constexpr int ctas = sizeof(T) == 4 ? k.ctas_f32 : k.ctas;
        f(I, ANY, norm_backward_kernel<T, k.vpt, k.warp, k.room, ctas, ANY>);
        f(I, WHOLE, norm_backward_kernel<T, k.vpt, k.warp, k.room, ctas, WHOLE>);
        f(I, ALL_GIVEN, norm_backward_kernel<T, k.vpt, k.warp, k.room, ctas, ALL_GIVEN>);
        each_back<T, I + 1>(f);
    }
}
template <typename T>
Given given(const NormArgs& a) {
    return !whole<T>(a) ? ANY : a.z.p && a.dy.p && a.dn.p && a.post && a.dx.p && a.dz.p && a.pre_w ? ALL_GIVEN : WHOLE;
}

template <typename T>
cudaError_t backward(const NormArgs& a, fe_dtype dtype, cudaStream_t st) {
    const int64_t nv = row_vecs(a.d, dtype);
    const NormForm form = backward_form(nv);
    const int threads = form_threads(form, nv);
    const int64_t workers = a.parts ? a.groups * a.parts : (a.groups + a.step - 1) / a.step;
    if (form == IN_PASSES) return launch_k(norm_backward_long_kernel<T>, dim3((unsigned)workers), dim3(threads), 0, st, false, a);
    const int i = back_kernel(form, threads);
    const int64_t ctas = form <= BY_WARP_2 ? (workers + kNormWarps - 1) / kNormWarps : workers;
    cudaError_t e = cudaSuccess;
    const Given g = given<T>(a);
    each_back<T, 0>([&](int k, Given of, auto kern) {
        if (k == i && of == g) e = launch_k(kern, dim3((unsigned)ctas), dim3(threads), back_smem(i), st, false, a, workers);
    });
    return e;
}

template <typename K>
cudaError_t allow(K kern, size_t bytes) {
    return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <typename T, int KIND>
cudaError_t prepare() {
    cudaError_t e;
    const size_t f = (kNormDepth + 1) * 2 * sizeof(uint4), f2 = 2 * f;
    if ((e = allow(norm_kernel<T, 1, false, 256, 4, KIND>, f * 256)) != cudaSuccess) return e;
    if ((e = allow(norm_kernel<T, 2, false, 192, 5, KIND>, f2 * 192)) != cudaSuccess) return e;
    if ((e = allow(norm_kernel<T, 2, false, 320, 3, KIND>, f2 * 320)) != cudaSuccess) return e;
    if ((e = allow(norm_kernel<T, 2, false, 512, 2, KIND>, f2 * 512)) != cudaSuccess) return e;
    return allow(norm_kernel<T, 2, false, kOne, 1, KIND>, f2 * kOne);
}

template <typename T>
cudaError_t prepare_backward() {
    cudaError_t e = cudaSuccess;
    int fit[kBacks] = {};
    each_back<T, 0>([&](int i, Given of, auto kern) {
        if (e != cudaSuccess || (e = allow(kern, back_smem(i))) != cudaSuccess) return;
        int per = 0;
        if ((e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kern, kBack[i].room, back_smem(i))) != cudaSuccess) return;
        fit[i] = of == ANY || per < fit[i] ? per : fit[i];
    });
    if (e == cudaSuccess) {  // (the same numbers for every handle)
        for (int i = 0; i < kBacks; ++i) back_fit[sizeof(T) == 4][i].store(fit[i], std::memory_order_relaxed);
    }
    return e;
}

template <typename T>
cudaError_t prepare_forward() {
    cudaError_t e = prepare<T, ANY>();
    if (e == cudaSuccess) e = prepare<T, WHOLE>();
    return e == cudaSuccess ? prepare<T, ALL_GIVEN>() : e;
}

}  // namespace

cudaError_t norm_prepare(fe_dtype dtype) { return dtype == FE_F32 ? prepare_forward<float>() : prepare_forward<bf16_t>(); }
cudaError_t norm_backward_prepare(fe_dtype dtype) { return dtype == FE_F32 ? prepare_backward<float>() : prepare_backward<bf16_t>(); }

int64_t norm_backward_plan(NormArgs& a, fe_dtype dtype, int num_sms) {
    const int64_t nv = row_vecs(a.d, dtype);
    const NormForm form = backward_form(nv);
    // workers that fill the GPU once
    const int i = form == IN_PASSES ? 0 : back_kernel(form, form_threads(form, nv));
    const int fit = form == IN_PASSES ? 1 : back_fit[dtype == FE_F32][i].load(std::memory_order_relaxed);
    const int64_t want = (int64_t)num_sms * (fit > 0 ? fit : kBack[i].ctas) * (form <= BY_WARP_2 ? kNormWarps : 1);
    const int64_t size = a.gate.p ? a.gate_rows : a.R;
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
