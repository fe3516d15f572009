// Log probabilities of given tokens with entropy and the most probable tokens, and their gradient
// (fe_token_logprobs). Bound by memory traffic: a row of logits is read once; with c = log2(e) / T
// and d = (x - m) c a thread keeps, of its elements,
//   m, S = sum 2^d, U = sum d 2^d,   so that   lse = m / T + log S,   H = log S - ln 2 U / S,
// against the largest m that its warp has seen, which four vectors of 16 bytes are compared with at a time.
//
// The K largest: of the threads' largest elements so far 32 groups are made; the K-th largest group maximum
// is no larger than the K-th largest element of the row, so elements that reach it are noted, and the few
// others are out. It is raised after 1, 3, 9, ... slices of a row. Rank among the notes is place in the
// result. Where there is not room for the notes (equal logits, or growing ones) the row is looked at again, by the
// final maxima, or the CTA takes out its largest element K times.
//
// Measured (GB300): 1568 rows of 128256 float32 logits with the ten largest 134 us (6.0 TB/s), 8189 rows of 32000
// bfloat16 102 us (5.1 TB/s; some 11 instructions an element), their gradient 152 us (6.9 TB/s).
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
constexpr int kLpThreads = 256;  // that read a row (four CTAs an SM)
constexpr float kLn2 = 0.6931471805599453f;

// order of (value, index): larger first by value (NaN above all, -0 equal to 0), then smaller index
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0xFFFFFFF0u;  // (so that no key is 2^64 - 1)
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t key_of(float x, uint32_t index) { return (uint64_t)order_of(x) << 32 | (uint32_t)~index; }
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return ~(uint32_t)k; }
// the element (not NaN) that a key was made of
__device__ __forceinline__ float key_value(uint64_t k) {
    const uint32_t u = (uint32_t)(k >> 32);
    return __uint_as_float((u & 0x80000000u) ? u & 0x7FFFFFFFu : ~u);
}

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
    // f(index) for a thread's loose elements; every pass over a share gives a thread the same elements
    template <typename F>
    __device__ __forceinline__ void each_loose(const F& f) const {
        for (int i = threadIdx.x; i < loose; i += kLpThreads) f(loose_at(i));
    }
    __device__ __forceinline__ int loose_at(int i) const { return i < head ? i : i + body; }
    __device__ __forceinline__ int index(int v) const { return head + v * V; }
    __device__ __forceinline__ uint4 load(int v) const { return reinterpret_cast<const uint4*>(p + head)[v]; }
    __device__ __forceinline__ uint4 load_once(int v) const { return __ldcs(reinterpret_cast<const uint4*>(p + head) + v); }
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

// what a sum of 2^d and of d 2^d with d = (x - m) c becomes against a larger maximum M: (u + t s) f and s f with
// t = (m - M) c, f = 2^t
__device__ __forceinline__ Stats rebased(Stats a, float M, float c) {
    const float t = (a.m - M) * c, f = ex2_approx(t);
    return Stats{M, a.s * f, f * fmaf(a.s, fmaxf(t, -1e4f), a.u)};
}
// the sum over a warp's lanes
__device__ __forceinline__ Stats warp_join(Stats a, float c) {
    a = rebased(a, warp_max(a.m), c);
    a.s = warp_sum(a.s);
    a.u = warp_sum(a.u);
    return a;
}
constexpr float kLowest = -3.402823466e38f;

// Room that a row's passes share.
struct LogprobShared {
    Stats stats[kLpThreads / 32];
    uint32_t best[kLpThreads / 32][32];  // order of the threads' largest elements, by warp
    uint64_t notes[kNotes];
    uint64_t top[kTopMax];
    uint32_t floor;
    int count, odd;
    Stats total;
};

// the largest key of a thread's share below `under`
template <typename T>
__device__ __forceinline__ uint64_t largest_below(const RowShare<T>& r, uint64_t under) {
    uint64_t best = 0;
    for (int v = r.v0 + threadIdx.x; v < r.v1; v += kLpThreads) {
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
    r.each_loose(one);
    return best;
}

// the reading warps, and the cluster; their lanes have to arrive as one, whatever branches lie before
__device__ __forceinline__ void lp_sync() {
    __syncwarp();
    named_sync(1, kLpThreads);
}
__device__ __forceinline__ void lp_cluster_sync(const cg::cluster_group& cluster) {
    __syncwarp();
    cluster.sync();
}

// The K-th largest of 32 groups' maxima (best: the order of the thread's largest element so far, 0 for none), which
// no more than K - 1 of the share's elements need exceed; 1, below every order, where fewer groups have any.
__device__ __forceinline__ uint32_t cta_floor(uint32_t best, int K, LogprobShared& sh) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    sh.best[warp][lane] = best;
    lp_sync();
    if (warp == 0) {
        uint32_t k = 0;
#pragma unroll
        for (int w = 0; w < kLpThreads / 32; ++w) k = max(k, sh.best[w][lane]);
        int rank = 0;  // among the 32 (equal ones by lane)
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const uint32_t o = __shfl_sync(0xffffffffu, k, i);
            rank += o > k || (o == k && i < lane);
        }
        if (rank == K - 1) sh.floor = max(k, 1u);
    }
    lp_sync();
    return sh.floor;
}
__device__ __forceinline__ void note(float x, int index, uint32_t floor, LogprobShared& sh) {
    if (order_of(x) >= floor) {
        const int at = atomicAdd(&sh.count, 1);
        if (at < kNotes) sh.notes[at] = key_of(x, index);
    }
}
// The K largest of the notes, sorted, into sh.top; false if there was not room for all.
__device__ __forceinline__ bool rank_notes(int K, LogprobShared& sh) {
    const int count = sh.count;
    if (count > kNotes) return false;
    for (int i = threadIdx.x; i < count; i += kLpThreads) {
        const uint64_t k = sh.notes[i];
        int rank = 0;
        for (int j = 0; j < count; ++j) rank += sh.notes[j] > k;
        if (rank < K) sh.top[rank] = k;
    }
    return true;
}

// The K largest keys of a CTA's share from a second look: at the threads whose largest element (best) reaches the
// floor of all, or, where that leaves too many, by taking out the largest K times.
template <typename T>
__device__ __forceinline__ void cta_top(const RowShare<T>& r, uint32_t best, int K, LogprobShared& sh) {
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, warps = kLpThreads / 32, step = kLpThreads;
    lp_sync();  // (the notes have been read)
    if (tid == 0) sh.count = 0;
    const uint32_t floor = cta_floor(best, K, sh);
    if (best >= floor) {
        for (int v = r.v0 + tid; v < r.v1; v += step) {
            float x[RowShare<T>::V];
            Vec16<T>::widen(r.load(v), x);
#pragma unroll
            for (int j = 0; j < RowShare<T>::V; ++j) note(x[j], r.index(v) + j, floor, sh);
        }
        const auto one = [&](int i) { note(load_one(r.p + i), i, floor, sh); };
        r.each_loose(one);
    }
    lp_sync();
    if (!rank_notes(K, sh)) {
        uint64_t under = ~(uint64_t)0, mine = under;  // (no key is that)
        for (int i = 0; i < K; ++i) {
            if (mine >= under) mine = largest_below(r, under);
            const uint64_t w = warp_max_key(mine);
            lp_sync();
            if (lane == 0) sh.notes[warp] = w;
            lp_sync();
            under = warp_max_key(lane < warps ? sh.notes[lane] : 0);
            if (tid == 0) sh.top[i] = under;
            if (under == 0) break;
        }
    }
}

// Slices of a row share on their way, by bulk copies of a warp that does nothing else: three of 16 KB a CTA, so
// that an SM's four CTAs have up to 192 KB outstanding, and the next row's first while a row is joined.
constexpr int kLpSlices = 3, kLpSlice = 4 * kLpThreads;  // vectors of a slice: four a thread
struct SliceBarriers {
    uint64_t full[kLpSlices], empty[kLpSlices];
};
template <typename T, bool TOP>
__global__ void __launch_bounds__(kLpThreads + 32, 4) logprob_kernel(const __grid_constant__ LogprobArgs a, float c, float inv_t) {
    constexpr int V = Vec16<T>::kN, B = kLpSlice / kLpThreads;
    extern __shared__ __align__(128) uint4 slices[];
    __shared__ LogprobShared sh;
    __shared__ SliceBarriers bar;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ranks = (int)cluster.num_blocks();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, warps = kLpThreads / 32, step = kLpThreads;
    const uint32_t nothing = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;  // minus infinity
    const int64_t row_step = gridDim.x / ranks;
    const auto share = [&](int64_t row) { return RowShare<T>((const T*)a.logits.p + row * a.logits.row, a.V, rank, ranks); };
    if (tid == 0) {
        for (int i = 0; i < kLpSlices; ++i) {
            mbar_init(&bar.full[i], 1);
            mbar_init(&bar.empty[i], kLpThreads / 32);
        }
        mbar_fence_init();
    }
    __syncthreads();
    int slot = 0;
    uint32_t phase = 0;  // of the slot's current use
    bool ok = true;      // (a wait that runs out is the last one: the kernel ends, its status says so)
    if (warp == warps) {  // ---- copies
        int n = 0;
        for (int64_t row = blockIdx.x / ranks; row < a.R; row += row_step) {
            if (lane == 0) {
                const RowShare<T> r = share(row);
                for (int v = r.v0; v < r.v1 && ok; v += kLpSlice, ++n) {
                    if (n >= kLpSlices && !(ok = mbar_wait(&bar.empty[slot], phase ^ 1, a.status))) break;
                    const uint32_t bytes = (uint32_t)min(kLpSlice, r.v1 - v) * 16;
                    mbar_arrive_expect_tx(&bar.full[slot], bytes);
                    bulk_g2s(slices + slot * kLpSlice, r.p + r.index(v), bytes, &bar.full[slot]);
                    if (++slot == kLpSlices) slot = 0, phase ^= 1;
                }
            }
            __syncwarp();
            if (ranks > 1) {
                lp_cluster_sync(cluster);
                lp_cluster_sync(cluster);
            }
        }
        if (lane == 0 && !ok) {  // (what is in flight lands before the CTA ends)
            for (int i = max(n - kLpSlices, 0); i < n; ++i) mbar_wait(&bar.full[i % kLpSlices], (uint32_t)(i / kLpSlices) & 1, a.status, 50000000LL);
        }
        return;
    }
    for (int64_t row = blockIdx.x / ranks; row < a.R; row += row_step) {
        const T* x0 = (const T*)a.logits.p + row * a.logits.row;
        const RowShare<T> r = share(row);
        // a token that is asked for, and its logit, are read ahead
        int id = -1;
        float xt = 0.f;
        if (rank == 0 && tid < a.J) {
            id = a.tokens[row * a.J + tid];
            if (id >= 0 && id < a.V) xt = load_one(x0 + id);
        }
        float m = kLowest, bx = -INFINITY;
        uint64_t s = 0, u = 0;  // by even and odd columns
        const uint64_t cc = pair_f32(c);
        const auto look = [&](const uint4* raw, int n) -> float {
            float top = largest<T>(raw[0]);
#pragma unroll
            for (int j = 1; j < B; ++j)
                if (j < n) top = fmaxf(top, largest<T>(raw[j]));
            if (TOP) bx = fmaxf(bx, top);
            if (__any_sync(0xffffffffu, top > m)) {
                const float M = warp_max(fmaxf(top, m)), t = (m - M) * c;
                const uint64_t f = pair_f32(ex2_approx(t));
                u = mul_x2(f, fma_x2(s, pair_f32(fmaxf(t, -1e4f)), u));
                s = mul_x2(f, s);
                m = M;
            }
            const uint64_t mm = pair_f32(-m);  // (-m c could be infinite where m is the lowest value)
#pragma unroll
            for (int j = 0; j < B; ++j) {
                if (j >= n) break;
                float x[V];
                Vec16<T>::widen(raw[j], x);
#pragma unroll
                for (int i = 0; i < V; i += 2) {
                    const uint64_t d = mul_x2(add_x2(pair_f32(__float_as_uint(x[i]), __float_as_uint(x[i + 1])), mm), cc);
                    const float dl = low_f32(d), dh = high_f32(d);
                    const uint64_t e = pair_f32(__float_as_uint(ex2_approx(dl)), __float_as_uint(ex2_approx(dh)));
                    s = add_x2(s, e);
                    u = fma_x2(e, pair_f32(__float_as_uint(fmaxf(dl, -1e4f)), __float_as_uint(fmaxf(dh, -1e4f))), u);
                }
            }
            return top;
        };
        uint32_t floor = 1;
        float reach = -INFINITY;  // the floor's value
        if (TOP) {
            if (tid == 0) sh.count = sh.odd = 0;
            if (tid < kTopMax) sh.top[tid] = 0;
            if (r.v0 >= r.v1) lp_sync();
        }
        int turn = 0, raise = 0;
        for (int v = r.v0; v < r.v1; v += kLpSlice, ++turn) {
            if (ok) ok = mbar_wait(&bar.full[slot], phase, a.status);
            const uint4* p = slices + slot * kLpSlice + tid;
            const int have = r.v1 - v - tid;
            uint4 raw[B];
#pragma unroll
            for (int j = 0; j < B; ++j) raw[j] = j * step < have ? p[j * step] : make_uint4(nothing, nothing, nothing, nothing);
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.empty[slot]);
            if (++slot == kLpSlices) slot = 0, phase ^= 1;
            const float top = look(raw, B);
            if (TOP) {
                if (turn == raise) {  // the floor, from the slices 0, 0 to 2, 0 to 8, ...
                    floor = cta_floor(r.v0 + tid < r.v1 ? order_of(bx) : 0, a.K, sh);
                    reach = floor < 0x00800000u ? -INFINITY : key_value((uint64_t)floor << 32);
                    raise = 3 * raise + 2;
                }
                if (top >= reach) {
#pragma unroll
                    for (int j = 0; j < B; ++j) {
                        if (j * step >= have) break;
                        float x[V];
                        Vec16<T>::widen(raw[j], x);
#pragma unroll
                        for (int i = 0; i < V; ++i) note(x[i], r.index(v + tid + j * step) + i, floor, sh);
                    }
                }
            }
        }
        for (int i = tid - lane; i < r.loose; i += step) {
            uint4 raw[1] = {make_uint4(nothing, nothing, nothing, nothing)};
            int at = -1;
            if (i + lane < r.loose) {
                at = r.loose_at(i + lane);
                raw[0].x = sizeof(T) == 2 ? (uint32_t) reinterpret_cast<const uint16_t*>(r.p)[at] | 0xFF800000u
                                          : reinterpret_cast<const uint32_t*>(r.p)[at];
            }
            const float top = look(raw, 1);
            if (TOP && at >= 0) note(top, at, floor, sh);
        }
        Stats st{m, warp_sum(low_f32(s) + high_f32(s)), warp_sum(low_f32(u) + high_f32(u))};
        if (TOP) {
            const float mine = low_f32(s) + high_f32(s);
            if (mine != mine) sh.odd = 1;  // NaN, or infinity, among a thread's elements
            lp_sync();
            if (sh.odd || !rank_notes(a.K, sh)) {
                uint32_t best = r.v0 + tid < r.v1 || tid < r.loose ? order_of(bx) : 0;
                if (mine != mine) best = (uint32_t)(largest_below(r, ~(uint64_t)0) >> 32);
                cta_top(r, best, a.K, sh);
            }
        }
        if (lane == 0) sh.stats[warp] = st;
        lp_sync();
        if (warp == 0) {
            st = warp_join(lane < warps ? sh.stats[lane] : Stats{kLowest, 0.f, 0.f}, c);
            if (lane == 0) sh.total = st;
        }
        if (ranks > 1) lp_cluster_sync(cluster);
        else lp_sync();
        if (rank == 0) {
            if (warp == 0 && ranks > 1) {
                st = warp_join(lane < ranks ? cluster.map_shared_rank(&sh, lane)->total : Stats{kLowest, 0.f, 0.f}, c);
                if (lane == 0) sh.stats[0] = st;
            }
            if (ranks > 1) {
                if (TOP) {  // the CTAs' lists, each of K sorted keys
                    const int all = ranks * a.K;
                    for (int i = tid; i < all; i += step) sh.notes[i] = cluster.map_shared_rank(&sh, i / a.K)->top[i % a.K];
                    lp_sync();
                    for (int i = tid; i < all; i += step) {
                        const uint64_t k = sh.notes[i];
                        int at = 0;
                        for (int j = 0; j < all; ++j) at += sh.notes[j] > k;
                        if (at < a.K && k) sh.top[at] = k;
                    }
                }
                lp_sync();
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
                float lp = 0.f;
                if (id >= a.V) atomicOr(a.status, ST_DEVICE);
                else if (id >= 0) lp = bad ? NAN : logp(xt);
                a.logprob[row * a.J + tid] = lp;
            }
            if (TOP && tid < a.K) {
                a.top_id[row * a.K + tid] = (int)key_index(sh.top[tid]);
                a.top_logprob[row * a.K + tid] = bad ? NAN : logp(key_value(sh.top[tid]));
            }
        }
        if (ranks > 1) lp_cluster_sync(cluster);  // (the others' shared memory has been read)
        else lp_sync();
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
                if (w + j * step < r.v1) next[j] = r.load_once(w + j * step);
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
        r.each_loose(one);
        __syncthreads();
        if (mine) store_one(g0 + id[tid], extra);
    }
}

template <typename T, bool TOP>
cudaError_t forward(const LogprobArgs& a, int num_sms, cudaStream_t st) {
    const int64_t vecs = a.V / Vec16<T>::kN;
    // CTAs of a row: the fewest rounds of CTAs (four an SM), counted in a thread's turns of four vectors, with some
    // four turns' time for a row's end and two for a cluster's
    const int threads = kLpThreads;
    int ranks = 1;
    int64_t best = 0;
    for (int r = 1; r <= 16 && (r == 1 || vecs >= (int64_t)r * threads); r *= 2) {
        const int64_t rounds = (a.R * r + num_sms * 4 - 1) / (num_sms * 4);
        const int64_t cost = rounds * ((vecs + r * threads * 4 - 1) / (r * threads * 4) + (r > 1 ? 6 : 4));
        if (!best || cost < best) {
            best = cost;
            ranks = r;
        }
    }
    const auto kern = logprob_kernel<T, TOP>;
    const float inv_t = 1.f / a.temperature;
    // CTAs that keep to one row each come and go; whole rows' CTAs stay, and have the next row on its way
    int64_t rows = ranks > 1 ? (int64_t)1 << 26 : (int64_t)num_sms * 4;
    if (rows > a.R) rows = a.R;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * ranks));
    cfg.blockDim = dim3(threads + 32);
    cfg.dynamicSmemBytes = kLpSlices * kLpSlice * sizeof(uint4);
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
    const int threads = kLpThreads;
    int shares = 1;
    while (a.R * shares * 2 <= num_sms * 4 && vecs >= (int64_t)shares * 2 * threads) shares *= 2;
    const int64_t units = a.R * shares, most = (int64_t)num_sms * 4;
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

cudaError_t logprobs_prepare(fe_dtype dtype) {
    const auto wide = [](auto kern) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        return e != cudaSuccess ? e : cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kLpSlices * kLpSlice * sizeof(uint4)));
    };
    const auto both = [&](auto a, auto b) {
        const cudaError_t e = wide(a);
        return e != cudaSuccess ? e : wide(b);
    };
    return dtype == FE_F32 ? both(logprob_kernel<float, true>, logprob_kernel<float, false>)
                           : both(logprob_kernel<bf16_t, true>, logprob_kernel<bf16_t, false>);
}

}  // namespace fe
