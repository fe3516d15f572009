// Log probabilities of given tokens with entropy and the most probable tokens, and their gradient
// (fe_token_logprobs). Bound by memory traffic: a row of logits is read once; with c = log2(e) / T
// and d = (x - m) c a thread keeps, of its elements,
//   m, S = sum 2^d, U = sum d 2^d,   so that   lse = m / T + log S,   H = log S - ln 2 U / S,
// rescaled when a vector of 16 bytes raises m, and the largest (value, index) that it saw.
//
// The K largest: of the threads' largest elements 32 groups are made; the K-th largest group maximum
// is no larger than the K-th largest element of the row, so the few threads whose maximum reaches it
// look through their elements again and note those that do. Rank among the notes is place in the
// result. Where more elements reach it than there is room for (a row whose large elements all fall
// to few threads), the CTA takes out its largest element K times instead.
//
// A cluster of 1 to 16 CTAs shares a row where there are too few rows to fill the GPU; its first CTA
// joins the others' results through distributed shared memory.
#include <cooperative_groups.h>

#include "fe_layer_common.cuh"

namespace fe {

namespace {

namespace cg = cooperative_groups;

constexpr int kTopMax = 32, kTokMax = 64;
constexpr int kNotes = 512;
constexpr int kLpThreads = 256;  // four CTAs an SM, each thread with up to eight vectors on their way or at hand
constexpr float kLn2 = 0.6931471805599453f;

// order of (value, index): larger first by value (NaN above all, -0 equal to 0), then smaller index
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0xFFFFFFF0u;  // (so that no key is 2^64 - 1)
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t key_of(float x, uint32_t index) { return (uint64_t)order_of(x) << 32 | (uint32_t)~index; }
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return ~(uint32_t)k; }

__device__ __forceinline__ uint64_t warp_max_key(uint64_t k) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const uint64_t v = __shfl_xor_sync(0xffffffffu, k, o);
        k = v > k ? v : k;
    }
    return k;
}

// The share of a row that CTA `rank` of `ranks` reads: vectors of 16 bytes [v0, v1) of the row's
// aligned body, and, rank 0, the elements before and behind the body.
template <typename T>
struct RowShare {
    static constexpr int V = Vec16<T>::kN;
    const T* p;
    int head, body, v0, v1, loose;  // elements before the body, in it; loose ones of this CTA
    __device__ __forceinline__ RowShare(const T* row, int n, int rank, int ranks) : p(row) {
        head = (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T);
        head = min(head, n);
        const int vecs = (n - head) / V;
        body = vecs * V;
        v0 = (int)((int64_t)vecs * rank / ranks);
        v1 = (int)((int64_t)vecs * (rank + 1) / ranks);
        loose = rank == 0 ? n - body : 0;
    }
    // f(index) for a thread's loose elements, those before the body and those behind it; every pass over a
    // share gives a thread the same elements
    template <typename F>
    __device__ __forceinline__ void each_before(const F& f) const {
        for (int i = threadIdx.x; i < min(head, loose); i += blockDim.x) f(i);
    }
    template <typename F>
    __device__ __forceinline__ void each_behind(const F& f) const {
        for (int i = head + threadIdx.x; i < loose; i += blockDim.x) f(i + body);
    }
    __device__ __forceinline__ int index(int v) const { return head + v * V; }
    __device__ __forceinline__ uint4 load(int v) const { return __ldcs(reinterpret_cast<const uint4*>(p + head) + v); }
};

struct Stats {
    float m, s, u;
};

// the largest element of a vector (NaN counts as nothing)
template <typename T>
__device__ __forceinline__ float largest(const uint4& x) {
    if (sizeof(T) == 4)
        return fmaxf(fmaxf(__uint_as_float(x.x), __uint_as_float(x.y)), fmaxf(__uint_as_float(x.z), __uint_as_float(x.w)));
    const auto max2 = [](uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    };
    const uint32_t m = max2(max2(x.x, x.y), max2(x.z, x.w));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
}

// d = (x - m) c against a larger maximum M: e^d becomes 2^t e^d with t = (m - M) c
__device__ __forceinline__ void rebase(Stats& a, float M, float c) {
    const float t = (a.m - M) * c, f = ex2_approx(t);
    a.u = f * fmaf(a.s, fmaxf(t, -1e4f), a.u);
    a.s *= f;
    a.m = M;
}
__device__ __forceinline__ void join(Stats& a, Stats b, float c) {
    const float M = fmaxf(a.m, b.m);
    rebase(a, M, c);
    rebase(b, M, c);
    a.s += b.s;
    a.u += b.u;
}

// Room that a row's passes share.
struct LogprobShared {
    Stats stats[32];
    uint64_t best[32][32];  // threads' largest keys, by warp
    uint64_t notes[kNotes];
    uint64_t top[kTopMax];
    uint64_t floor;
    int count;
    Stats total;
};

// the largest key of a thread's share below `under`
template <typename T>
__device__ __forceinline__ uint64_t largest_below(const RowShare<T>& r, uint64_t under) {
    uint64_t best = 0;
    for (int v = r.v0 + threadIdx.x; v < r.v1; v += blockDim.x) {
        float x[RowShare<T>::V];
        Vec16<T>::widen(r.load(v), x);
#pragma unroll
        for (int i = 0; i < RowShare<T>::V; ++i) {
            const uint64_t k = key_of(x[i], r.index(v) + i);
            if (k < under && k > best) best = k;
        }
    }
    const auto one = [&](int i) {
        const uint64_t k = key_of(load_one(r.p + i), i);
        if (k < under && k > best) best = k;
    };
    r.each_before(one);
    r.each_behind(one);
    return best;
}

// The K largest keys of a CTA's share, sorted, into sh.top (0 where the share has fewer).
template <typename T>
__device__ __forceinline__ void cta_top(const RowShare<T>& r, uint64_t best, int K, LogprobShared& sh) {
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, warps = blockDim.x / 32;
    sh.best[warp][lane] = best;
    if (tid == 0) sh.count = 0;
    __syncthreads();
    if (warp == 0) {
        uint64_t k = 0;
        for (int w = 0; w < warps; ++w) k = max(k, sh.best[w][lane]);
        // rank of a group's maximum among the 32 (equal ones, of empty groups, by lane)
        int rank = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const uint64_t o = __shfl_sync(0xffffffffu, k, i);
            rank += o > k || (o == k && i < lane);
        }
        if (rank == K - 1) sh.floor = k;
        sh.top[lane] = 0;
    }
    __syncthreads();
    const uint64_t floor = max(sh.floor, (uint64_t)1);
    if (best >= floor) {
        const auto note = [&](float x, int index) {
            const uint64_t k = key_of(x, index);
            if (k >= floor) {
                const int at = atomicAdd(&sh.count, 1);
                if (at < kNotes) sh.notes[at] = k;
            }
        };
        const int step = blockDim.x;
        int v = r.v0 + tid;
        for (; v + 3 * step < r.v1; v += 4 * step) {
            uint4 raw[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) raw[j] = r.load(v + j * step);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float x[RowShare<T>::V];
                Vec16<T>::widen(raw[j], x);
#pragma unroll
                for (int i = 0; i < RowShare<T>::V; ++i) note(x[i], r.index(v + j * step) + i);
            }
        }
        for (; v < r.v1; v += step) {
            float x[RowShare<T>::V];
            Vec16<T>::widen(r.load(v), x);
#pragma unroll
            for (int i = 0; i < RowShare<T>::V; ++i) note(x[i], r.index(v) + i);
        }
        const auto one = [&](int i) { note(load_one(r.p + i), i); };
        r.each_before(one);
        r.each_behind(one);
    }
    __syncthreads();
    const int count = sh.count;
    if (count <= kNotes) {
        for (int i = tid; i < count; i += blockDim.x) {
            const uint64_t k = sh.notes[i];
            int rank = 0;
            for (int j = 0; j < count; ++j) rank += sh.notes[j] > k;
            if (rank < K) sh.top[rank] = k;
        }
    } else {
        uint64_t under = ~(uint64_t)0;  // (no key: an index is below 2^30)
        uint64_t mine = best;
        for (int i = 0; i < K; ++i) {
            if (mine >= under) mine = largest_below(r, under);
            const uint64_t w = warp_max_key(mine);
            __syncthreads();
            if (lane == 0) sh.notes[warp] = w;
            __syncthreads();
            under = warp_max_key(lane < warps ? sh.notes[lane] : 0);
            if (tid == 0) sh.top[i] = under;
            if (under == 0) break;
        }
    }
    __syncthreads();
}

template <typename T, bool TOP>
__global__ void __launch_bounds__(kLpThreads, 4) logprob_kernel(const __grid_constant__ LogprobArgs a, float c, float inv_t) {
    constexpr int V = Vec16<T>::kN;
    __shared__ LogprobShared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ranks = (int)cluster.num_blocks();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, warps = blockDim.x / 32;
    for (int64_t row = blockIdx.x / ranks; row < a.R; row += gridDim.x / ranks) {
        const T* x0 = (const T*)a.logits.p + row * a.logits.row;
        const RowShare<T> r(x0, a.V, rank, ranks);
        Stats st{-3.402823466e38f, 0.f, 0.f};
        float bx = -INFINITY;  // the largest element and its index
        int bi = -1;
        // n elements (a whole vector, or one)
        const auto take = [&](const uint4& raw, int n, int index) {
            float x[V];
            Vec16<T>::widen(raw, x);
            const float top = n == V ? largest<T>(raw) : x[0];
            if (top > st.m) rebase(st, top, c);
            if (n == V) {
                const uint64_t cc = pair_f32(c), mm = pair_f32(-st.m);  // (-m c could be infinite where m is the lowest value)
                uint64_t s = 0, u = 0;
#pragma unroll
                for (int i = 0; i < V / 2; ++i) {
                    const uint64_t d = mul_x2(add_x2(pair_f32(__float_as_uint(x[2 * i]), __float_as_uint(x[2 * i + 1])), mm), cc);
                    const float dl = low_f32(d), dh = high_f32(d);
                    const uint64_t e = pair_f32(__float_as_uint(ex2_approx(dl)), __float_as_uint(ex2_approx(dh)));
                    s = add_x2(s, e);
                    u = fma_x2(e, pair_f32(__float_as_uint(fmaxf(dl, -1e4f)), __float_as_uint(fmaxf(dh, -1e4f))), u);
                }
                st.s += low_f32(s) + high_f32(s);
                st.u += low_f32(u) + high_f32(u);
            } else {
                const float d = (x[0] - st.m) * c, e = ex2_approx(d);
                st.s += e;
                st.u = fmaf(e, fmaxf(d, -1e4f), st.u);
            }
            if (TOP && (top > bx || bi < 0)) {
                bx = top;
                bi = index;
#pragma unroll
                for (int i = V - 1; i >= 0; --i)
                    if (i < n && x[i] == top) bi = index + i;
            }
        };
        const int step = blockDim.x;
        const auto one = [&](int i) { take(make_uint4(sizeof(T) == 2 ? (uint32_t) reinterpret_cast<const uint16_t*>(r.p)[i]
                                                                     : reinterpret_cast<const uint32_t*>(r.p)[i], 0, 0, 0), 1, i); };
        r.each_before(one);  // (by growing index, so that the first of equal elements is kept)
        // four vectors of a thread in flight, the next four requested before these are looked at
        int v = r.v0 + tid;
        uint4 next[4];
        const auto request = [&](int w) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (w + j * step < r.v1) next[j] = r.load(w + j * step);
        };
        request(v);
        for (; v < r.v1; v += 4 * step) {
            uint4 raw[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) raw[j] = next[j];
            request(v + 4 * step);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (v + j * step < r.v1) take(raw[j], V, r.index(v + j * step));
        }
        r.each_behind(one);
        uint64_t best = 0;
        if (TOP) {
            if (bi >= 0) best = key_of(bx, bi);
            if (st.s != st.s) best = largest_below(r, ~(uint64_t)0);  // NaN among a thread's elements: its first one
            cta_top(r, best, a.K, sh);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            Stats b;
            b.m = __shfl_xor_sync(0xffffffffu, st.m, o);
            b.s = __shfl_xor_sync(0xffffffffu, st.s, o);
            b.u = __shfl_xor_sync(0xffffffffu, st.u, o);
            join(st, b, c);
        }
        if (lane == 0) sh.stats[warp] = st;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < warps; ++w) join(st, sh.stats[w], c);
            sh.total = st;
        }
        if (ranks > 1) cluster.sync();
        else __syncthreads();
        if (rank == 0) {
            if (tid == 0 && ranks > 1) {
                st = sh.total;
                for (int k = 1; k < ranks; ++k) join(st, cluster.map_shared_rank(&sh, k)->total, c);
                sh.stats[0] = st;
            }
            if (ranks > 1) {
                if (TOP) {  // the CTAs' lists, each of K sorted keys
                    const int all = ranks * a.K;
                    for (int i = tid; i < all; i += step) sh.notes[i] = cluster.map_shared_rank(&sh, i / a.K)->top[i % a.K];
                    __syncthreads();
                    for (int i = tid; i < all; i += step) {
                        const uint64_t k = sh.notes[i];
                        int at = 0;
                        for (int j = 0; j < all; ++j) at += sh.notes[j] > k;
                        if (at < a.K && k) sh.top[at] = k;
                    }
                }
                __syncthreads();
            }
            st = ranks > 1 ? sh.stats[0] : sh.total;
            // a row of nothing but -inf: S = 0
            const bool none = st.s == 0.f;
            const float base = st.m, logs = none ? 0.f : logf(st.s);
            const auto logp = [&](float x) { return none ? -INFINITY : (x - base) * inv_t - logs; };
            if (tid == 0) {
                if (a.stats) {
                    a.stats[2 * row] = base;
                    a.stats[2 * row + 1] = none ? -INFINITY : logs;
                }
                if (a.lse) a.lse[row] = none ? -INFINITY : base * inv_t + logs;
                if (a.entropy) a.entropy[row] = none ? 0.f : logs - kLn2 * (st.u / st.s);
            }
            const bool bad = st.s != st.s;
            if (tid < a.J) {
                const int id = a.tokens[row * a.J + tid];
                float lp = 0.f;
                if (id >= a.V) atomicOr(a.status, ST_DEVICE);
                else if (id >= 0) lp = bad ? NAN : logp(load_one(x0 + id));
                a.logprob[row * a.J + tid] = lp;
            }
            if (TOP && tid < a.K) {
                const int id = (int)key_index(sh.top[tid]);
                const bool there = id >= 0 && id < a.V;  // (always)
                a.top_id[row * a.K + tid] = id;
                a.top_logprob[row * a.K + tid] = bad || !there ? NAN : logp(load_one(x0 + id));
            }
        }
        if (ranks > 1) cluster.sync();  // (the others' shared memory has been read)
        else __syncthreads();
    }
}

// One CTA a share of a row: dl = (1 / T) p (A - dH (log p + H)) + (1 / T) (what the row's tokens get),
// A = dlse - sum of the tokens' gradients.
template <typename T>
__global__ void __launch_bounds__(kLpThreads, 4) logprob_backward_kernel(const __grid_constant__ LogprobArgs a, float c, float inv_t, int shares) {
    constexpr int V = Vec16<T>::kN;
    __shared__ int id[kTokMax + kTopMax];
    __shared__ float coef[kTokMax + kTopMax];
    __shared__ float total;
    const int tid = threadIdx.x, n = a.J + a.K;
    const int64_t units = a.R * shares;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int64_t row = unit / shares;
        const T* x0 = (const T*)a.logits.p + row * a.logits.row;
        T* g0 = (T*)a.dlogits.p + row * a.dlogits.row;
        const RowShare<T> r(x0, a.V, (int)(unit % shares), shares);
        // the first vectors are on their way while the row's tokens are read
        const int step = blockDim.x;
        int v = r.v0 + tid;
        uint4 next[4];
        const auto request = [&](int w) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (w + j * step < r.v1) next[j] = r.load(w + j * step);
        };
        request(v);
        __syncthreads();
        if (tid < n) {
            int t;
            float d;
            if (tid < a.J) {
                t = a.tokens[row * a.J + tid];
                if (t >= a.V) atomicOr(a.status, ST_DEVICE);
                d = a.dlogprob && t >= 0 && t < a.V ? a.dlogprob[row * a.J + tid] : 0.f;
                if (!a.dlogprob) t = -1;
            } else {
                t = a.dtop ? a.top_in[row * a.K + tid - a.J] : -1;
                d = t >= 0 && t < a.V ? a.dtop[row * a.K + tid - a.J] : 0.f;
            }
            if (t >= a.V) t = -1;
            id[tid] = t;
            coef[tid] = d;
        }
        __syncthreads();
        if (tid < 32) {
            float s = 0.f;
            for (int i = tid; i < n; i += 32) s += coef[i];
            s = warp_sum(s);
            if (tid == 0) total = s;
        }
        // log p = (x - base) / T - log S: the two apart, as their sum may round away what matters
        const float base = a.stats_in[2 * row];
        float logs = a.stats_in[2 * row + 1];
        const float dh = a.dentropy ? a.dentropy[row] : 0.f;
        const float h = a.dentropy ? a.entropy_in[row] : 0.f;
        if (logs == -INFINITY) logs = 0.f;  // (every p is 0 then)
        const float logs2 = logs * kLog2e;
        __syncthreads();
        const float A = ((a.dlse ? a.dlse[row] : 0.f) - total - dh * h) * inv_t, B = -dh * kLn2 * inv_t;
        const auto grad = [&](float x) {
            const float d = fmaf(x - base, c, -logs2), p = ex2_approx(d);
            return p * fmaf(B, fmaxf(d, -1e4f), A);
        };
        // the tokens of this share: what they have besides, before the logits may be overwritten
        float extra = 0.f;
        bool mine = false;
        if (tid < n && id[tid] >= 0) {
            const int t = id[tid], b = t - r.head;
            mine = b >= 0 && b < r.body ? b / V >= r.v0 && b / V < r.v1 : r.loose > 0;
            for (int i = 0; i < tid && mine; ++i) mine = id[i] != t;
            if (mine) {
                float s = 0.f;
                for (int i = tid; i < n; ++i) s += id[i] == t ? coef[i] : 0.f;
                extra = grad(load_one(x0 + t)) + s * inv_t;
            }
        }
        __syncthreads();
        const bool aligned = (((uintptr_t)(g0 + r.head)) & 15) == 0;
        const auto put = [&](int w, const uint4& raw) {
            float x[V];
            Vec16<T>::widen(raw, x);
            const uint64_t cc = pair_f32(c), mm = pair_f32(-base), lc = pair_f32(-logs2), A2 = pair_f32(A), B2 = pair_f32(B);
#pragma unroll
            for (int i = 0; i < V; i += 2) {
                const uint64_t d = fma_x2(add_x2(pair_f32(__float_as_uint(x[i]), __float_as_uint(x[i + 1])), mm), cc, lc);
                const float dl = low_f32(d), dh = high_f32(d);
                const uint64_t p = pair_f32(__float_as_uint(ex2_approx(dl)), __float_as_uint(ex2_approx(dh)));
                const uint64_t q = fma_x2(B2, pair_f32(__float_as_uint(fmaxf(dl, -1e4f)), __float_as_uint(fmaxf(dh, -1e4f))), A2);
                const uint64_t y = mul_x2(p, q);
                x[i] = low_f32(y);
                x[i + 1] = high_f32(y);
            }
            T* g = g0 + r.index(w);
            if (aligned) {
                __stcs(reinterpret_cast<uint4*>(g), pack16<T>(x));
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) store_one(g + i, x[i]);
            }
        };
        for (; v < r.v1; v += 4 * step) {
            uint4 raw[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) raw[j] = next[j];
            request(v + 4 * step);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (v + j * step < r.v1) put(v + j * step, raw[j]);
        }
        const auto one = [&](int i) { store_one(g0 + i, grad(load_one(x0 + i))); };
        r.each_before(one);
        r.each_behind(one);
        __syncthreads();
        if (mine) store_one(g0 + id[tid], extra);
    }
}

template <typename T, bool TOP>
cudaError_t forward(const LogprobArgs& a, int num_sms, cudaStream_t st) {
    const int64_t vecs = a.V / Vec16<T>::kN;
    // CTAs of a row: as many as still leave a thread four vectors, until the GPU has four CTAs an SM
    int ranks = 1, threads = kLpThreads;
    while (ranks < 16 && a.R * ranks * 2 <= num_sms * 4 && vecs >= (int64_t)ranks * 2 * threads) ranks *= 2;
    while (threads > 128 && ranks == 1 && vecs < threads * 2) threads /= 2;
    const auto kern = logprob_kernel<T, TOP>;
    const float inv_t = 1.f / a.temperature;
    int64_t rows = (int64_t)num_sms * (1024 / threads);  // as many CTAs as fit at once
    if (rows > a.R) rows = a.R;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * ranks));
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ranks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, a, kLog2e * inv_t, inv_t);
}

template <typename T>
cudaError_t backward(const LogprobArgs& a, int num_sms, cudaStream_t st) {
    const int64_t vecs = a.V / Vec16<T>::kN;
    int shares = 1, threads = kLpThreads;
    while (a.R * shares * 2 <= num_sms * 4 && vecs >= (int64_t)shares * 2 * threads) shares *= 2;
    while (threads > 128 && vecs < (int64_t)shares * threads * 2) threads /= 2;
    const int64_t units = a.R * shares, most = (int64_t)num_sms * (1024 / threads);
    const float inv_t = 1.f / a.temperature;
    return launch_k(logprob_backward_kernel<T>, dim3((unsigned)(units < most ? units : most)), dim3(threads), 0, st, false, a,
                    kLog2e * inv_t, inv_t, shares);
}

}  // namespace

cudaError_t launch_token_logprobs(const LogprobArgs& a, fe_dtype dtype, int num_sms, cudaStream_t st) {
    if (dtype == FE_F32) return a.K ? forward<float, true>(a, num_sms, st) : forward<float, false>(a, num_sms, st);
    return a.K ? forward<bf16_t, true>(a, num_sms, st) : forward<bf16_t, false>(a, num_sms, st);
}

cudaError_t launch_token_logprobs_backward(const LogprobArgs& a, fe_dtype dtype, int num_sms, cudaStream_t st) {
    return dtype == FE_F32 ? backward<float>(a, num_sms, st) : backward<bf16_t>(a, num_sms, st);
}

cudaError_t logprobs_prepare() {
    cudaError_t e;
    const auto wide = [](auto kern) { return cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1); };
    if ((e = wide(logprob_kernel<float, true>)) != cudaSuccess || (e = wide(logprob_kernel<float, false>)) != cudaSuccess) return e;
    if ((e = wide(logprob_kernel<bf16_t, true>)) != cudaSuccess) return e;
    return wide(logprob_kernel<bf16_t, false>);
}

}  // namespace fe
