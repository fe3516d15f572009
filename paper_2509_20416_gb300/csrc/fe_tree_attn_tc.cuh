// Attention over the cache on the 5th-generation tensor cores (tcgen05, TMEM), for bfloat16
// queries over bfloat16 or e4m3 caches.
//
// With r query rows sharing a KV head (nodes x grouped heads), a cached row of 2 hd elements is
// used in 4 hd r operations: about r / 2 operations a byte from bfloat16, r from e4m3, against
// ~290 that the GPU can do per byte it reads. So up to about a hundred rows the kernel is bound
// by reading the cache once, above that by the tensor cores and the exponentials; a single
// design serves both ends.
//
// A CTA (one per SM, persistent; fe_attn_plan.cuh divides the work) runs two streams, each with
// its own 128 x 128 score block S_g and 128 x hd output block O_g in TMEM (2 x (128 + 128)
// columns, all 512). An item of more than 128 rows gives each stream 128 of them, and both use
// every key/value tile; a smaller one gives both streams the same rows, on alternate tiles, and
// adds their results at the end. While one stream's softmax runs on the CUDA cores, the tensor
// cores work on the other's products.
//   warps 0-3, 4-7   softmax of stream 0, 1: thread = row (TMEM lane)
//   warps 8-11       loaders: rows from the cache into 128-byte-swizzled tiles of 128 slots (K and
//                    V alike, [slot][hd]), by cp.async, or converted from e4m3 on the way
//   warp 12          issues the MMAs: S = Q K^T (K-major operands), O += P V with P (bfloat16)
//                    read from TMEM over S's own columns and V as the MN-major operand
//   warp 13          e4m3: bulk copies of the raw rows (runs of rows are contiguous in a page)
// The softmax keeps a reference maximum per row and rescales O only when the maximum has grown by
// more than 2^8 (the probabilities then stay below 2^8, where bfloat16 is as precise as below 1):
// after the first tiles that is rare, and it saves a pass over O per tile. Sums and statistics
// are float32; probabilities are rounded to bfloat16 for the second product, which costs 2^-9 of
// each on average and is what the 16-bit tensor path offers.
// Values in slots that a row does not see meet a zero probability, but 0 x NaN is NaN: the loaders
// zero the non-finite elements of nodes' value rows and flag the segment, whose epilogue then
// adds their terms to the rows that do see them.
#pragma once

#include "fe_attn_plan.cuh"
#include "fe_stream.cuh"
#include "fe_tc.cuh"

namespace fe {

constexpr int kTcTile = 128;
using TcPlan = Plan<kAttnItemRows, kTcTile, true>;

// MT: 128-row query blocks a CTA must hold (1 when no item has more than 128 rows)
template <int HD, bool Q8, int MT>
struct TcShape {
    static constexpr int kTileBytes = kTcTile * HD * 2;  // also a query block's
    static constexpr int kRawBytes = kTcTile * HD;
    static constexpr int kSlots = Q8 ? 4 : 7 - MT;           // tiles in flight
    static constexpr int kRawSlots = Q8 ? (MT == 1 ? 4 : 2) : 0;
    static constexpr int kThreads = Q8 ? 448 : 416;
    static constexpr int kData = MT * kTileBytes + kSlots * kTileBytes + kRawSlots * kRawBytes;
};

struct TcState {
    uint64_t full[6], empty[6], rawfull[4], rawempty[4], qfull, qempty, sfull[2], pfull[2], odone, ofree, mlfull, mlfree,
        drain;
    uint32_t tmem;
    int abort;
    int odd[8];        // by segment: non-finite value elements were set aside
    float2 ml[128];    // stream 1's (maximum, sum) for the join of the two streams
};

template <int HD, bool Q8, int MT>
constexpr int tc_smem() { return 1024 + TcShape<HD, Q8, MT>::kData + (int)sizeof(TcState); }

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool valid) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// MN-major operand block of 128 K-rows x hd: 128-byte-swizzled atoms of 8 rows x 64 elements,
// 1024 bytes between 8-row groups (K), `half` bytes between 64-element groups (MN)
__device__ __forceinline__ uint64_t sw128_desc_mn(uint32_t smem_addr, uint32_t half) {
    return sw128_desc(smem_addr) | ((uint64_t)(half >> 4) << 16);
}

// D[tmem] (+)= A[tmem, bf16 pairs] * B[smem desc], one M x N x 16 step
__device__ __forceinline__ void tc_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                          uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// The slots of [s0, s0 + 32) that node `node` sees, as bits.
__device__ __forceinline__ uint32_t seen_bits(const TreeAttnArgs& a, const Segment& g, int node, int s0) {
    const int P = g.s.P;
    auto ones = [](int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; };
    if (!a.mask) return ones(min(P + node + 1, g.end) - s0);
    uint32_t w = ones(P - s0);
    const uint8_t* row = a.mask + ((int64_t)g.b * a.T + node) * a.T - P + s0;
    const int lo = max(P - s0, 0), hi = min(g.end - s0, 32);
    for (int j0 = lo; j0 < hi; j0 += 8) {  // eight loads at a time
        uint8_t v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = j0 + k < hi ? row[j0 + k] : 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) w |= v[k] ? 1u << ((j0 + k) & 31) : 0u;
    }
    return w;
}

// ---- loaders ------------------------------------------------------------------------------------
// What a lane knows of its row (32 w + lane) of a tile: the cache row, or -1 for a slot past the
// item's end (or with a bad page id); and the row's scales.
struct RowInfo {
    int64_t row;
    float ks, vs;
};

template <bool Q8>
__device__ __forceinline__ RowInfo row_info(const TreeAttnArgs& a, const Segment& g, int tile, int r) {
    RowInfo x{-1, 0.f, 0.f};
    const int64_t slot = (int64_t)tile * kTcTile + r;
    int64_t row;
    if (tile < g.t1 && slot < g.end && cache_row(a.cache, g.b, slot, row, a.status)) {
        x.row = row + g.h * head_step(a.cache);
        if (Q8) {
            x.ks = a.cache.ks[x.row];
            x.vs = a.cache.vs[x.row];
        }
    }
    return x;
}

// Query rows of block `blk` into a swizzled K-major tile (rows past the item's are zero).
template <int HD>
__device__ __forceinline__ void load_q(const TreeAttnArgs& a, const Segment& g, int blk, unsigned char* dst, int w, int lane) {
    constexpr int CH = HD / 8, RP = 32 / CH;  // 16-byte chunks a row, rows a warp access
    const int r0 = g.m * kAttnItemRows + blk * 128 + w * 32 + lane;
    const bf16_t* src = nullptr;
    if (r0 < g.rows)
        src = (const bf16_t*)a.q.p + g.b * a.q.batch + (int64_t)(r0 / a.G) * a.q.token +
              (int64_t)(g.h * a.G + r0 % a.G) * a.q.head;
    const int c = lane % CH;
#pragma unroll 4
    for (int i = 0; i < 32 / RP; ++i) {
        const int r = i * RP + lane / CH;
        const bf16_t* p = (const bf16_t*)__shfl_sync(0xffffffffu, (unsigned long long)src, r);
        unsigned char* d = dst + (c >> 3) * 16384 + sw128_offset(w * 32 + r, c & 7);
        if (a.q_vec) {
            cp_async16(smem_u32(d), p ? p + c * 8 : (const bf16_t*)a.q.p, p != nullptr);
        } else {
            uint32_t x[4] = {0, 0, 0, 0};
            if (p)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = (uint32_t)p[c * 8 + 2 * e].bits | (uint32_t)p[c * 8 + 2 * e + 1].bits << 16;
            *reinterpret_cast<uint4*>(d) = make_uint4(x[0], x[1], x[2], x[3]);
        }
    }
}

// one tile of bf16 rows
template <int HD>
__device__ __forceinline__ void load_tile(const void* base, const RowInfo& x, unsigned char* dst, int w, int lane) {
    constexpr int CH = HD / 8, RP = 32 / CH;
    const int c = lane % CH;
#pragma unroll
    for (int i = 0; i < 32 / RP; ++i) {
        const int r = i * RP + lane / CH;
        const int64_t row = __shfl_sync(0xffffffffu, x.row, r);
        const char* src = (const char*)base + ((row < 0 ? 0 : row) * HD + c * 8) * 2;
        cp_async16(smem_u32(dst + (c >> 3) * 16384 + sw128_offset(w * 32 + r, c & 7)), src, row >= 0);
    }
}

// Zero the non-finite elements of a lane's own chunks of a value tile, in rows from `first` on.
template <int HD>
__device__ __forceinline__ bool scrub_tile(unsigned char* tile, int first, int w, int lane) {
    constexpr int CH = HD / 8, RP = 32 / CH;
    const int c = lane % CH;
    bool odd = false;
#pragma unroll 4
    for (int i = 0; i < 32 / RP; ++i) {
        const int r = w * 32 + i * RP + lane / CH;
        if (r < first) continue;
        uint32_t* d = reinterpret_cast<uint32_t*>(tile + (c >> 3) * 16384 + sw128_offset(r, c & 7));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t u = d[e];
            uint32_t keep = 0xffffffffu;
            if ((u & 0x7F80u) == 0x7F80u) keep &= 0xffff0000u;
            if ((u & 0x7F800000u) == 0x7F800000u) keep &= 0x0000ffffu;
            if (keep != 0xffffffffu) {
                d[e] = u & keep;
                odd = true;
            }
        }
    }
    return odd;
}

// One tile of e4m3 rows, converted: raw [128][HD] bytes to bf16 values number * scale (exact for
// power-of-two scales). Rows without a cache row become zero; in rows from `first` on, so do
// non-finite elements (returns whether there were any).
template <int HD>
__device__ __forceinline__ bool convert_tile(const unsigned char* raw, int64_t row_of_lane, float scale_of_lane, int first,
                                             unsigned char* dst, int w, int lane) {
    constexpr int CH = HD / 16, RP = 32 / CH;
    const int c = lane % CH;
    bool odd = false;
#pragma unroll 4
    for (int i = 0; i < 32 / RP; ++i) {
        const int rr = i * RP + lane / CH, r = w * 32 + rr;
        const bool valid = __shfl_sync(0xffffffffu, row_of_lane, rr) >= 0;
        const float s = __shfl_sync(0xffffffffu, scale_of_lane, rr);
        uint4 u = *reinterpret_cast<const uint4*>(raw + r * HD + c * 16);
        if (!valid) u = make_uint4(0, 0, 0, 0);
        const uint32_t in[4] = {u.x, u.y, u.z, u.w};
        uint32_t o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 f = e4m3x2_to_f32(in[e / 2] >> (16 * (e & 1)));
            o[e] = pack_bf16(f.x * s, f.y * s);
        }
        if (!valid) {  // (0 times a stale scale may be NaN)
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = 0;
        } else if (r >= first) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if ((o[e] & 0x7F80u) == 0x7F80u) { o[e] &= 0xffff0000u; odd = true; }
                if ((o[e] & 0x7F800000u) == 0x7F800000u) { o[e] &= 0x0000ffffu; odd = true; }
            }
        }
        // two 16-byte chunks; lanes of the upper half of a 128-byte-row pair go in the other order,
        // so that eight lanes store into different banks
        unsigned char* base = dst + (c >> 2) * 16384;
        const int c0 = 2 * (c & 3);
        const uint4 lo = make_uint4(o[0], o[1], o[2], o[3]), hi = make_uint4(o[4], o[5], o[6], o[7]);
        const bool swap = (c >> 2) != 0;
        *reinterpret_cast<uint4*>(base + sw128_offset(r, swap ? c0 + 1 : c0)) = swap ? hi : lo;
        *reinterpret_cast<uint4*>(base + sw128_offset(r, swap ? c0 : c0 + 1)) = swap ? lo : hi;
    }
    return odd;
}

// Ring positions of a segment's tiles. They are loaded in the order of their first use:
// K0 K1 V0 K2 V1 ... K(n-1) V(n-2) V(n-1).
__device__ __forceinline__ int pos_k(int t) { return t == 0 ? 0 : 2 * t - 1; }
__device__ __forceinline__ int pos_v(int t, int n) { return t < n - 1 ? 2 * t + 2 : 2 * n - 1; }

// ---- the kernel -----------------------------------------------------------------------------------
template <int HD, bool Q8, int MT>
__global__ void __launch_bounds__(TcShape<HD, Q8, MT>::kThreads, 1) tree_attn_tc_kernel(const TreeAttnArgs a) {
    using SH = TcShape<HD, Q8, MT>;
    constexpr int S = SH::kSlots, RS = Q8 ? SH::kRawSlots : 1, TB = SH::kTileBytes;
    extern __shared__ unsigned char dsm_raw[];
    unsigned char* qbuf = (unsigned char*)(((uintptr_t)dsm_raw + 1023) & ~(uintptr_t)1023);
    unsigned char* ring = qbuf + MT * TB;
    unsigned char* rawring = ring + S * TB;
    TcState& st = *reinterpret_cast<TcState*>(qbuf + SH::kData);
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const PlanArgs pa = plan_args(a);
    griddep_launch_dependents();

    bool bad = false;
    SegmentWalk<TcPlan> walk;
    walk.init(pa, blockIdx.x, gridDim.x, &bad);
    if (bad && blockIdx.x == 0 && warp == 0) atomicOr(a.status, ST_CAPACITY);
    if (walk.done) return;  // (the same in every warp)

    if (t == 0) {
        for (int i = 0; i < S; ++i) {
            mbar_init(&st.full[i], 128);
            mbar_init(&st.empty[i], 1);
        }
        for (int i = 0; i < RS; ++i) {
            mbar_init(&st.rawfull[i], 1);
            mbar_init(&st.rawempty[i], 128);
        }
        mbar_init(&st.qfull, 128);
        mbar_init(&st.qempty, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&st.sfull[i], 1);
            mbar_init(&st.pfull[i], 4);
        }
        mbar_init(&st.odone, 1);
        mbar_init(&st.ofree, 8);
        mbar_init(&st.mlfull, 4);
        mbar_init(&st.mlfree, 4);
        mbar_init(&st.drain, 1);
        st.abort = 0;
        for (int i = 0; i < 8; ++i) st.odd[i] = 0;
        mbar_fence_init();
    }
    if (warp == 12) tc_alloc(&st.tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = st.tmem;
    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait_abortable(bar, parity & 1u, a.status, &st.abort); };
    Segment g;

    if (warp >= 8 && warp < 12) {  // ---- loaders
        const int w = warp - 8;
        uint32_t i = 0, sig = 0;  // tiles issued, tiles announced
        uint32_t qpos = 0xffffffffu;  // the tile whose group also brings the queries
        uint32_t seg = 0;
        bool ok = true;
        // announce tiles up to (not including) `upto`, whose copies are complete
        auto announce = [&](uint32_t upto) {
            if (sig == upto) return;
            fence_async_proxy();
            for (; sig != upto; ++sig) {
                if (sig == qpos) mbar_arrive(&st.qfull);
                mbar_arrive(&st.full[sig % S]);
            }
        };
        auto slot_free = [&]() -> bool {
            if (i < (uint32_t)S) return true;
            uint64_t* e = &st.empty[i % S];
            const uint32_t par = (i / S - 1) & 1u;
            if (!Q8 && !mbar_try_wait(e, par)) {
                // everything is in flight or in use: announce what is here before blocking
                cp_async_wait<0>();
                announce(i);
            }
            return wait(e, par);
        };
        while (ok && walk.next(pa, g)) {
            if (seg > 0) {  // the queries' buffer is free once the last segment's scores are done
                if (!mbar_try_wait(&st.qempty, (seg - 1) & 1u)) {
                    cp_async_wait<0>();
                    announce(i);
                }
                if (!(ok = wait(&st.qempty, seg - 1))) break;
            }
            const int nt = g.t1 - g.t0;
            RowInfo x0 = row_info<Q8>(a, g, g.t0, w * 32 + lane), x1 = row_info<Q8>(a, g, g.t0 + 1, w * 32 + lane), x2 = x1;
            for (int b = 0; b < g.weight; ++b) load_q<HD>(a, g, b, qbuf + b * TB, w, lane);
            qpos = i;
            // key or value tile tt (from this segment's first) of the rows in x
            auto load = [&](bool val, int tt, const RowInfo& x) {
                unsigned char* dst = ring + (i % S) * TB;
                const int first = g.s.P - (g.t0 + tt) * kTcTile;  // first row of the tile that is a node's
                if constexpr (Q8) {
                    const uint32_t rs = i % RS;
                    if (i == qpos) {  // (the queries' copies)
                        cp_async_commit();
                        cp_async_wait<0>();
                    }
                    if (!(ok = wait(&st.rawfull[rs], i / RS)) || !(ok = slot_free())) return;
                    const bool odd = convert_tile<HD>(rawring + rs * SH::kRawBytes, x.row, val ? x.vs : x.ks,
                                                      val ? first : kTcTile, dst, w, lane);
                    if (odd) st.odd[seg & 7] = 1;
                    mbar_arrive(&st.rawempty[rs]);
                    ++i;
                    announce(i);
                } else {
                    if (!(ok = slot_free())) return;
                    load_tile<HD>(val ? a.cache.v : a.cache.k, x, dst, w, lane);
                    cp_async_commit();
                    ++i;
                    if (val && first < kTcTile) {
                        cp_async_wait<0>();
                        if (scrub_tile<HD>(dst, first, w, lane)) st.odd[seg & 7] = 1;
                        announce(i);
                    } else {
                        cp_async_wait<2>();
                        if (i - sig > 2) announce(i - 2);
                    }
                }
            };
            load(false, 0, x0);
            for (int tt = 0; tt < nt && ok; ++tt) {
                if (tt + 1 < nt) {
                    x2 = row_info<Q8>(a, g, g.t0 + tt + 2, w * 32 + lane);
                    load(false, tt + 1, x1);
                    if (!ok) break;
                }
                load(true, tt, x0);
                x0 = x1;
                x1 = x2;
            }
            ++seg;
        }
        cp_async_wait<0>();
        if (ok) announce(i);
    } else if (warp == 12) {  // ---- MMA issuer
        const uint32_t id_qk = idesc_bf16_f32(128, kTcTile);
        const uint32_t id_pv = idesc_bf16_f32(128, HD) | (1u << 16);  // B is MN-major
        uint32_t base = 0, seg = 0, np[2] = {0, 0};
        bool ok = true;
        while (walk.next(pa, g)) {
            if (lane == 0 && ok) {
                const int nt = g.t1 - g.t0;
                const bool pair = g.weight == 2;
                const int n = pair ? 2 * nt : nt;
                auto qk = [&](int j) {
                    const int gs = j & 1, tt = pair ? j >> 1 : j;
                    const uint32_t p = base + pos_k(tt);
                    if (j == 0 && !(ok = wait(&st.qfull, seg))) return;
                    if (!(ok = wait(&st.full[p % S], p / S))) return;
                    tc_fence_after();
                    const uint32_t qa = smem_u32(qbuf + (pair ? gs * TB : 0)), ka = smem_u32(ring + (p % S) * TB);
#pragma unroll
                    for (int k = 0; k < HD / 16; ++k)
                        tc_mma(tmem + gs * 128, sw128_desc(qa + (k >> 2) * 16384) + 2 * (k & 3),
                               sw128_desc(ka + (k >> 2) * 16384) + 2 * (k & 3), id_qk, k ? 1u : 0u);
                    if (!pair || gs == 1) tc_commit(&st.empty[p % S]);
                    tc_commit(&st.sfull[gs]);
                    if (j == n - 1) tc_commit(&st.qempty);
                };
                qk(0);
                if (ok && n > 1) qk(1);
                for (int j = 0; j < n && ok; ++j) {
                    const int gs = j & 1, tt = pair ? j >> 1 : j;
                    const uint32_t p = base + pos_v(tt, nt);
                    if (!(ok = wait(&st.pfull[gs], np[gs]))) break;
                    ++np[gs];
                    if (j == 0 && seg > 0 && !(ok = wait(&st.ofree, seg - 1))) break;
                    if (!(ok = wait(&st.full[p % S], p / S))) break;
                    tc_fence_after();
                    const uint32_t va = smem_u32(ring + (p % S) * TB);
#pragma unroll
                    for (int k = 0; k < kTcTile / 16; ++k)
                        tc_mma_ts(tmem + 256 + gs * 128, tmem + gs * 128 + k * 8, sw128_desc_mn(va + k * 2048, 16384), id_pv,
                                  j > 1 || k ? 1u : 0u);
                    if (!pair || gs == 1) tc_commit(&st.empty[p % S]);
                    if (j + 2 < n) qk(j + 2);
                }
                if (ok) tc_commit(&st.odone);
                base += 2 * nt;
            }
            ++seg;
            __syncwarp();
        }
        // every MMA issued has finished reading shared memory and TMEM before the CTA ends
        if (lane == 0) {
            tc_commit(&st.drain);
            mbar_wait(&st.drain, 0, a.status, 100000000LL);
        }
        __syncwarp();
    } else if (Q8 && warp == 13) {  // ---- raw rows of an e4m3 cache
        uint32_t i = 0;
        bool ok = true;
        while (ok && walk.next(pa, g)) {
            const int nt = g.t1 - g.t0;
            for (int l = 0; l < 2 * nt && ok; ++l, ++i) {
                const bool val = l == 2 * nt - 1 || (l > 0 && !(l & 1));
                const int tt = l == 0 ? 0 : l == 2 * nt - 1 ? nt - 1 : val ? (l - 2) / 2 : (l + 1) / 2;
                const uint32_t rs = i % RS;
                if (i >= (uint32_t)RS && !(ok = wait(&st.rawempty[rs], i / RS - 1))) break;
                const int s0 = (g.t0 + tt) * kTcTile, s1 = min(s0 + kTcTile, g.end);
                const int ps = a.cache.page_size ? a.cache.page_size : a.cache.max_seq;
                const int p0 = s0 / ps, np = (s1 - 1) / ps - p0 + 1;
                // a lane's runs: pages p0 + lane, + 32, ...
                auto run = [&](int k, int& from, int& rows, int64_t& row) -> bool {
                    const int lo = max(s0, (p0 + k) * ps), hi = min((int64_t)s1, (int64_t)(p0 + k + 1) * ps);
                    from = lo - s0;
                    rows = hi - lo;
                    if (!cache_row(a.cache, g.b, lo, row, a.status)) return false;
                    row += g.h * head_step(a.cache);
                    return true;
                };
                int from, rows, bytes = 0;
                int64_t row;
                for (int k = lane; k < np; k += 32)
                    if (run(k, from, rows, row)) bytes += rows * HD;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) bytes += __shfl_xor_sync(0xffffffffu, bytes, o);
                if (lane == 0) mbar_arrive_expect_tx(&st.rawfull[rs], bytes);
                __syncwarp();
                unsigned char* dst = rawring + rs * SH::kRawBytes;
                const char* src = (const char*)(val ? a.cache.v : a.cache.k);
                for (int k = lane; k < np; k += 32)
                    if (run(k, from, rows, row)) bulk_g2s(dst + from * HD, src + row * HD, rows * HD, &st.rawfull[rs]);
            }
        }
        // leave with no copy in flight: the last tiles have landed
        for (uint32_t j = i > (uint32_t)RS ? i - RS : 0; j < i; ++j) mbar_wait(&st.rawfull[j % RS], (j / RS) & 1u, a.status);
    } else if (warp < 8) {  // ---- softmax
        const int gs = warp >> 2, wl = warp & 3;
        const uint32_t lanes = (uint32_t)(wl * 32) << 16;
        const uint32_t ts = tmem + gs * 128 + lanes, to = tmem + 256 + gs * 128 + lanes;
        const float scale2 = a.scale * kLog2e;
        uint32_t ns = 0, nj = 0, seg = 0;  // score blocks taken, joins, segments
        bool ok = true;
        while (walk.next(pa, g)) {
            const int nt = g.t1 - g.t0;
            const bool pair = g.weight == 2;
            const int row = g.m * kAttnItemRows + (pair ? gs * 128 : 0) + wl * 32 + lane;  // of the item's head
            const int node = row / a.G;
            const bool live = row < g.rows;
            const bool idle = g.m * kAttnItemRows + (pair ? gs * 128 : 0) + wl * 32 >= g.rows;  // the whole warp
            float m = -INFINITY, sum = 0.f;  // reference maximum (log2 units), sum of 2^(s - m)
            for (int tt = pair ? 0 : gs; tt < nt && ok; tt += pair ? 1 : 2) {
                const int tile = g.t0 + tt;
                if (!(ok = wait(&st.sfull[gs], ns))) break;
                ++ns;
                tc_fence_after();
                if (!idle) {
                    const bool tail = (tile + 1) * kTcTile > g.s.P;  // some slots need the mask
                    uint32_t see[4] = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
                    if (tail) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) see[c] = live ? seen_bits(a, g, node, tile * kTcTile + 32 * c) : 0u;
                    }
                    float mx = -INFINITY;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float s[32];
                        tc_ld32(ts + 32 * c, s);
                        if (tail) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) s[e] = see[c] >> e & 1u ? s[e] : -INFINITY;
                        }
#pragma unroll
                        for (int e = 0; e < 32; ++e) mx = fmaxf(mx, s[e]);
                    }
                    mx = mx == -INFINITY ? -INFINITY : mx * scale2;
                    const bool first = tt < 2 && (tt == 0 || !pair);
                    if (first) {
                        m = mx;
                    } else if (__any_sync(0xffffffffu, mx > m + 8.f)) {
                        const float mn = fmaxf(m, mx), f = mn == -INFINITY ? 1.f : exp2f(m - mn);
                        sum *= f;
                        m = mn;
#pragma unroll
                        for (int c = 0; c < HD; c += 16) {
                            float o[16];
                            uint32_t u[16];
                            tc_ld16(to + c, o);
#pragma unroll
                            for (int e = 0; e < 16; ++e) u[e] = __float_as_uint(o[e] * f);
                            tc_st16(to + c, u);
                        }
                    }
                    const float ms = m == -INFINITY ? 0.f : m;
                    float z0 = 0.f, z1 = 0.f;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float s[32];
                        uint32_t u[16];
                        tc_ld32(ts + 32 * c, s);
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float p0 = ex2_approx(fmaf(s[e], scale2, -ms)), p1 = ex2_approx(fmaf(s[e + 1], scale2, -ms));
                            if (tail) {
                                p0 = see[c] >> e & 1u ? p0 : 0.f;
                                p1 = see[c] >> (e + 1) & 1u ? p1 : 0.f;
                            }
                            z0 += p0;
                            z1 += p1;
                            u[e / 2] = pack_bf16(p0, p1);
                        }
                        tc_st16(ts + 16 * c, u);
                    }
                    sum += z0 + z1;
                    tc_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&st.pfull[gs]);
            }
            // ---- the segment's result
            ok = ok && wait(&st.odone, seg);
            if (ok) {
                tc_fence_after();
                float f0 = 1.f, f1 = 0.f;  // weights of this stream's block, and of stream 1's (alternating)
                const bool join = !pair && nt > 1;
                if (join && gs == 1) {
                    if (nj > 0 && !(ok = wait(&st.mlfree, nj - 1))) break;
                    st.ml[wl * 32 + lane] = make_float2(m, sum);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&st.mlfull);
                } else if (join) {
                    if (!(ok = wait(&st.mlfull, nj))) break;
                    const float2 o = st.ml[wl * 32 + lane];
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&st.mlfree);
                    const float mn = fmaxf(m, o.x), ms = mn == -INFINITY ? 0.f : mn;
                    f0 = exp2f(m - ms);
                    f1 = exp2f(o.x - ms);
                    sum = sum * f0 + o.y * f1;
                    m = mn;
                }
                nj += join;
                if (!idle && (pair || gs == 0)) {
                    const bool odd = *(volatile int*)&st.odd[seg & 7] != 0;
                    const int head = g.h * a.G + row % a.G;
                    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
                    const int64_t pr = ((int64_t)blockIdx.x * 2 + g.slot) * kAttnItemRows + (row - g.m * kAttnItemRows);
#pragma unroll 1
                    for (int c = 0; c < HD; c += 32) {
                        float o[32];
                        tc_ld32(to + c, o);
                        if (join) {
                            float p[32];
                            tc_ld32(to + 128 + c, p);
                            // (a stream without any visible slot has zero sums: its block counts for nothing)
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = o[e] * f0 + p[e] * f1;
                        }
                        if (live && odd) {  // terms of non-finite value elements, for the nodes that see them
                            const bf16_t* q = (const bf16_t*)a.q.p + g.b * a.q.batch + (int64_t)node * a.q.token +
                                              (int64_t)head * a.q.head;
                            for (int s = max(g.s.P, g.t0 * kTcTile); s < min(g.end, g.t1 * kTcTile); ++s) {
                                const RowInfo x = row_info<Q8>(a, g, s / kTcTile, s % kTcTile);
                                if (x.row < 0 || !(seen_bits(a, g, node, s) & 1u)) continue;
                                auto at = [&](const void* p, float sc, int e) {
                                    if (Q8) {
                                        const float f = e4m3x2_to_f32(((const uint8_t*)p)[x.row * HD + e]).x;
                                        return bf16_to_f32((uint16_t)pack_bf16(f * sc, 0.f));
                                    }
                                    return Storage<bf16_t>::load((const bf16_t*)p, x.row * HD + e);
                                };
                                bool any = false;
                                for (int e = 0; e < 32; ++e) any |= !finite_f32(at(a.cache.v, x.vs, c + e));
                                if (!any) continue;
                                float dot = 0.f;
                                for (int e = 0; e < HD; ++e) dot = fmaf(Storage<bf16_t>::load(q, e), at(a.cache.k, x.ks, e), dot);
                                const float p = exp2f(dot * scale2 - (m == -INFINITY ? 0.f : m));
#pragma unroll
                                for (int e = 0; e < 32; ++e) {
                                    const float v = at(a.cache.v, x.vs, c + e);
                                    if (!finite_f32(v)) o[e] += p * v;
                                }
                            }
                        }
                        if (live && g.whole) {
                            bf16_t* dst = (bf16_t*)a.out.p + g.b * a.out.batch + (int64_t)node * a.out.token +
                                          (int64_t)head * a.out.head + c;
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = sum == 0.f ? 0.f : o[e] * inv;
                            if (a.out_vec) {
#pragma unroll
                                for (int e = 0; e < 32; e += 8) *reinterpret_cast<uint4*>(dst + e) = pack16<bf16_t>(o + e);
                            } else {
#pragma unroll
                                for (int e = 0; e < 32; ++e) store_one(dst + e, o[e]);
                            }
                        } else if (live) {
                            float4* dst = reinterpret_cast<float4*>(a.part_o + pr * HD + c);
#pragma unroll
                            for (int e = 0; e < 8; ++e) dst[e] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                        }
                        __syncwarp();
                    }
                    if (live) {
                        if (!g.whole)
                            *reinterpret_cast<float2*>(a.part_ml + 2 * pr) = make_float2(m, sum);
                        else if (a.lse)
                            a.lse[((int64_t)g.b * a.T + node) * a.H + head] =
                                sum == 0.f ? -INFINITY : m * 0.6931471805599453f + logf(sum);
                    }
                }
                tc_fence_before();
                __syncwarp();
                // (the loaders are at most two segments ahead, the other stream at most one behind)
                if (gs == 0 && wl == 0 && lane == 0) st.odd[(seg + 4) & 7] = 0;
                if (lane == 0) mbar_arrive(&st.ofree);
            }
            ++seg;
            if (!ok) break;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 12) tc_dealloc(tmem, 512);
}

}  // namespace fe
