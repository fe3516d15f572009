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
//   warps 0-3, 4-7   softmax of stream 0, 1: thread = row (TMEM lane); they also load the queries
//                    that TMA cannot, the next segment's while this one's last product runs, split
//                    them for e4m3 keys, and write the results
//   warps 8-11       loaders. bfloat16: values of tiles with nodes are looked through where TMA put
//                    them, tiles that TMA does not bring come by cp.async. e4m3: a tile's key scales,
//                    and values converted to bfloat16 [slot][hd]
//   warps 12, 13     issue the MMAs of stream 0, 1: S = Q K^T (K-major operands), O += P V with P
//                    (bfloat16) read from TMEM over S's own columns and V as the MN-major operand
//   warp 14          plans: the CTA's segments (shares of items), a few ahead of their use, and their
//                    queries by TMA where heads and strides allow
//   warp 15          TMA: tiles in boxes of a page's rows into the rings; e4m3 values by bulk copies
// e4m3 keys go to the tensor cores as they are, with queries as two e4m3 parts (split_query_row);
// their scales are applied to the scores.
//
// The softmax keeps a reference per row, its maximum rounded up to a whole power of two, and rescales
// O (exactly, therefore) only when the maximum has grown by more than 2^12: after the first tiles that
// is rare, and it saves a pass over O per tile and a pass over the scores for their maximum. The
// probabilities then stay below 2^12, where floating point is as precise as below 1, and sums over a
// long cache are far from overflow. (81 nodes over 131k e4m3 slots: 362 us with 2^8, 353 with 2^12,
// 354 with 2^16 or 2^24.) Sums and statistics are float32. The probabilities are rounded to bfloat16
// for the second product, up to 2^-8 of each and without a bias: outputs are off by 2.3e-3 of their
// size against 64 bits, by 1.7e-3 from their own rounding alone. Two parts a probability would double
// that product, half of the tensor cores' work. A row's sum is that of the unrounded ones: the log-
// sum-exp needs it to 32 bits. 2^x is ex2.approx's, off by up to 2^-22.
// Values in slots that a row does not see meet a zero probability, but 0 x NaN is NaN: the loaders
// zero the non-finite elements of nodes' value rows (and of what lies past the item's end) and flag
// the segment, whose epilogue then adds their terms to the rows that do see them.
//
// What bounds it (GB300, 128-wide heads): 32 sequences over 256 to 4096 bfloat16 slots, 8 KV heads,
// 17 nodes x 4 heads: 67 us, 4.4 TB/s (pages of 16: 77); 49 x 4 rows: 86 us, 660 TFLOP/s. 81 nodes x
// 64 heads over 131k slots: bfloat16 299 us, 1160 TFLOP/s; e4m3 358 us, 972 TFLOP/s. The long ones
// are bound by a stream's chain, softmax (1300 clocks a tile; with key scales 2700) after product
// after softmax, of which two are in flight; the products alone need 2048 of the 3150 clocks that a
// tile pair takes. No pipe of the softmax is near its limit: over 2 x 1021 tokens the exponentials' is
// used to 26 % (32 a clock and SM: 512 clocks a tile), the integer pipe to 35 %, the issue slots to
// 43 %. The short ones pay 7 us of start (schedule, first tile, cold instruction caches) and an
// epilogue of 2 us a share of an item.
#pragma once

#include <cuda.h>

#include "fe_attn_plan.cuh"
#include "fe_stream.cuh"
#include "fe_tc.cuh"

namespace fe {

constexpr float kRescale = 12.f;  // log2 of the growth of a row's maximum that its block is rescaled for
// Key tiles whose scales are at hand. A softmax still reads tile t's when the loaders may be at tile
// t + 1 + kKeySlots (the other stream's products may be one tile further).
constexpr int kTcScales = 8;
// MT: 128-row query blocks a CTA must hold (1 when no item has more than 128 rows)
template <int HD, bool Q8, int MT>
struct TcShape {
    static constexpr int kTileBytes = kTcTile * HD * 2;  // bfloat16 tile; also a query block's
    static constexpr int kRawBytes = kTcTile * HD;       // e4m3 tile
    // tiles in flight: bfloat16 keys and values in one ring; e4m3 keys as they are, raw values, and
    // converted values in three
    static constexpr int kSlots = Q8 ? 2 : MT == 1 ? 6 : 5;
    static constexpr int kKeySlots = Q8 ? 3 : 0;
    static constexpr int kRawSlots = Q8 ? (MT == 1 ? 3 : 2) : 0;
    // the key tiles' scales, and the query rows' [segment parity][block][row]
    static constexpr int kScaleBytes = Q8 ? (kTcScales + 4) * kTcTile * 4 : 0;
    static constexpr int kThreads = 512;
    static constexpr int kReaders = 15;  // warps that read the segments
    static constexpr int kData = MT * kTileBytes + kSlots * kTileBytes + (kKeySlots + kRawSlots) * kRawBytes + kScaleBytes;
};

constexpr int kTcSegs = 4;  // segments planned ahead

struct TcState {
    uint64_t full[6], empty[6], landed[6], kfull[4], kempty[4], rawfull[4], rawempty[4], segfull[kTcSegs], segempty[kTcSegs], qfull, qempty, qready, sfull[2],
        pfull[2], odone[2], ofree, mlfull, mlfree, drain[2], turn[2];
    Segment seg[kTcSegs];  // weight 0: no more
    uint32_t tmem;
    int abort;
    int odd[8];        // by segment: non-finite value elements were set aside
    float2 ml[2][128];  // the streams' (maximum, sum), for their join
};

template <int HD, bool Q8, int MT>
constexpr int tc_smem() {
    constexpr int bytes = TcShape<HD, Q8, MT>::kData + (int)sizeof(TcState);
    static_assert(bytes <= 227 * 1024, "shared memory of a CTA");
    return bytes;
}

__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// one arrival on `bar` once all cp.async of this thread so far are complete
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// arrive on `bar` n times
__device__ __forceinline__ void mbar_arrive_n(uint64_t* bar, uint32_t n) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(n) : "memory");
}

// one box of a 3-D tensor map to shared memory, its bytes counted on `bar`
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
        : "memory");
}

// true in one lane of a converged warp (the same lane every time)
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

// MN-major operand block of 128 K-rows x hd: 128-byte-swizzled atoms of 8 rows x 64 elements,
// 1024 bytes between 8-row groups (K), `half` bytes between 64-element groups (MN)
__device__ __forceinline__ uint64_t sw128_desc_mn(uint32_t smem_addr, uint32_t half) {
    return sw128_desc(smem_addr) | ((uint64_t)(half >> 4) << 16);
}

// e4m3 operands: the key tile's descriptor (64-byte swizzle for 64-wide heads: mode 4, 512 bytes
// between 8-row groups), the instruction descriptor (float32 from e4m3 and e4m3, K-major) and one
// M x N x 32 step
template <int HD>
__device__ __forceinline__ uint64_t key_desc(uint32_t smem_addr) {
    if (HD == 128) return sw128_desc(smem_addr);
    return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | (uint64_t)(512u >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)4 << 61;
}
constexpr uint32_t idesc_e4m3_f32(int M, int N) { return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24); }
__device__ __forceinline__ void tc_mma_e4m3(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
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
__device__ __forceinline__ void st_global_32(void* p, const uint32_t (&w)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                 "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// The slow part of a warp's bounded wait, one call, not a copy at every place: until the phase is
// complete, another role gives up, or the time is over (which it then tells the others and the host).
// It has failed if it failed in any lane.
__device__ __noinline__ bool tc_wait_slow(uint64_t* bar, uint32_t parity, int* status, int* abort, int64_t budget_ns) {
    const uint64_t t0 = globaltimer_ns();
    bool done = false;
    while (!(done = mbar_try_wait(bar, parity)) && !*(volatile int*)abort) {
        if ((int64_t)(globaltimer_ns() - t0) > budget_ns) {
            atomicOr(status, ST_TIMEOUT);
            *(volatile int*)abort = 1;
        }
    }
    return __all_sync(0xffffffffu, done);
}
// What a wait is allowed besides, for each tile that it lasts: several times a tile's time.
constexpr int64_t kTileBudgetNs = 20000;

// The slots of [s0, s0 + 128) that node `node` sees, as bits (x: the first 64).
__device__ __noinline__ ulonglong2 seen_bits(const TreeAttnArgs& a, const Segment& g, int node, int s0) {
    const int P = g.s.P;
    auto ones = [](int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull; };
    if (!a.mask) {
        const int n = min(P + node + 1, g.end) - s0;
        return make_ulonglong2(ones(n), ones(n - 64));
    }
    const int lo = max(P - s0, 0), hi = min(g.end - s0, kTcTile);  // the nodes' slots in the tile
    // their bytes, in aligned words (the first and last may hold up to three neighbouring bytes)
    const uint8_t* row = a.mask + ((int64_t)g.b * a.T + node) * a.T - P + s0;  // slot s0's byte
    ulonglong2 w = make_ulonglong2(0ull, 0ull);
    int c = lo - (int)((uintptr_t)(row + lo) & 3);  // a word's first slot
#pragma unroll 1
    for (; c < hi; c += 32) {
        uint32_t v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = c + 4 * k < hi ? *reinterpret_cast<const uint32_t*>(row + c + 4 * k) : 0u;
        uint32_t bits = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {  // bytes that are not zero
            const uint32_t z = (((v[k] & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | v[k]) >> 7 & 0x01010101u;
            bits |= (z * 0x01020408u >> 24) << (4 * k);
        }
        const unsigned long long b = bits;
        if (c < 0) w.x |= b >> -c;
        else if (c < 64) w.x |= b << c;
        else w.y |= b << (c - 64);
        if (c > 32 && c < 64) w.y |= b >> (64 - c);
    }
    // (bits below the first node's slot came from neighbouring bytes: those slots are the prefix's)
    return make_ulonglong2((w.x & ones(hi)) | ones(lo), (w.y & ones(hi - 64)) | ones(lo - 64));
}

// ---- loaders ------------------------------------------------------------------------------------
// What a lane knows of its row (32 w + lane) of a tile: the cache row, or -1 for a slot past the
// item's end (or with a bad page id); the row's scales; and whether it is a node's. A node's row may
// be hidden from all and hold anything. A NaN or infinity among its scales would spread through a
// masked score or a zero probability: unless valid_scale, a key's scale becomes 1 and a value row
// zeros. (Looked at where they are used: here it would wait for the loads.)
struct RowInfo {
    int64_t row;
    float ks, vs;
    bool node;
};
__device__ __forceinline__ bool valid_scale(float x) { return __float_as_uint(x) - (7u << 23) <= 240u << 23; }

template <bool Q8>
__device__ __forceinline__ RowInfo row_info(const TreeAttnArgs& a, const Segment& g, int tile, int r) {
    RowInfo x{-1, 0.f, 0.f, false};
    const int64_t slot = (int64_t)tile * kTcTile + r;
    int64_t row;
    if (tile < g.t1 && slot < g.end && cache_row(a.cache, g.b, slot, row, a.status)) {
        x.row = row + g.h * head_step(a.cache);
        if (Q8) {
            x.ks = a.cache.ks[x.row];
            x.vs = a.cache.vs[x.row];
            x.node = slot >= g.s.P;
        }
    }
    return x;
}

// A warp's 32 query rows (rows r0 ..) into rows w * 32 .. of a swizzled K-major tile; rows past
// the item's are zero.
template <int HD>
__device__ __noinline__ void load_q(const TreeAttnArgs& a, const Segment& g, int r0, unsigned char* dst, int w, int lane) {
    constexpr int CH = HD / 8, RP = 32 / CH;  // 16-byte chunks a row, rows a warp access
    const int c = lane % CH, row = r0 + lane;
    unsigned long long mine = 0;
    if (row < g.rows)
        mine = (unsigned long long)((const bf16_t*)a.q.p + g.b * a.q.batch + (int64_t)(row / a.G) * a.q.token +
                                    (int64_t)(g.h * a.G + row % a.G) * a.q.head);
    const uint32_t d = smem_u32(dst) + (c >> 3) * 16384 + w * 4096;
#pragma unroll 2
    for (int i = 0; i < 32 / RP; ++i) {
        const int r = i * RP + lane / CH;
        const unsigned long long src = __shfl_sync(0xffffffffu, mine, r);
        if (a.q_vec) {
            cp_async16(d + sw128_offset(r, c & 7), (const void*)((src ? src : (unsigned long long)a.q.p) + (src ? c * 16 : 0)), src != 0);
        } else {
            uint32_t x[4] = {0, 0, 0, 0};
            const bf16_t* p = (const bf16_t*)src;
            if (p)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = (uint32_t)p[c * 8 + 2 * e].bits | (uint32_t)p[c * 8 + 2 * e + 1].bits << 16;
            *reinterpret_cast<uint4*>(dst + (c >> 3) * 16384 + w * 4096 + sw128_offset(r, c & 7)) = make_uint4(x[0], x[1], x[2], x[3]);
        }
    }
}

// one tile of bf16 rows
template <int HD>
__device__ __forceinline__ void load_tile(const void* base, const RowInfo& x, unsigned char* dst, int w, int lane) {
    constexpr int CH = HD / 8, RP = 32 / CH;
    const int c = lane % CH;
    const unsigned long long mine = x.row < 0 ? 0ull : (unsigned long long)base + (unsigned long long)x.row * (HD * 2);
    const uint32_t d = smem_u32(dst) + (c >> 3) * 16384 + w * 4096;
#pragma unroll 4
    for (int i = 0; i < 32 / RP; ++i) {
        const int r = i * RP + lane / CH;
        const unsigned long long src = __shfl_sync(0xffffffffu, mine, r);
        cp_async16(d + sw128_offset(r, c & 7), (const void*)((src ? src : (unsigned long long)base) + c * 16), src != 0);
    }
}

// Byte offset of 16-byte chunk c of row r in an e4m3 key tile: K-major rows of HD bytes, 128-byte
// swizzled, or 64-byte swizzled for 64-wide heads
template <int HD>
__device__ __forceinline__ uint32_t key_offset(int r, int c) {
    return HD == 128 ? sw128_offset(r, c) : (uint32_t)(r * 64 + ((c ^ (r >> 1 & 3)) << 4));
}

// one key tile of e4m3 rows as they are
template <int HD>
__device__ __forceinline__ void load_key_tile(const void* base, const RowInfo& x, unsigned char* dst, int w, int lane) {
    constexpr int CH = HD / 16, RP = 32 / CH;
    const int c = lane % CH;
    const unsigned long long mine = x.row < 0 ? 0ull : (unsigned long long)base + (unsigned long long)x.row * HD;
#pragma unroll 2
    for (int i = 0; i < 32 / RP; ++i) {
        const int r = i * RP + lane / CH;
        const unsigned long long src = __shfl_sync(0xffffffffu, mine, r);
        cp_async16(smem_u32(dst) + key_offset<HD>(w * 32 + r, c), (const void*)((src ? src : (unsigned long long)base) + c * 16), src != 0);
    }
}

// Zero the non-finite elements of a lane's own chunks of a value tile, in rows from `first` on;
// whether there were any. Looking comes first, by a short loop (exponent bits all ones carry into
// the sign bit); the repair is rare.
template <int HD>
__device__ __noinline__ bool repair_tile(unsigned char* tile, int first, int w, int lane) {
    constexpr int CH = HD / 8, RP = 32 / CH;
    const int c = lane % CH;
    bool odd = false;
#pragma unroll 1
    for (int i = 0; i < 32 / RP; ++i) {
        const int r = w * 32 + i * RP + lane / CH;
        uint32_t* d = reinterpret_cast<uint32_t*>(tile + (c >> 3) * 16384 + sw128_offset(r, c & 7));
#pragma unroll 1
        for (int e = 0; e < 4 && r >= first; ++e) {
            uint32_t u = d[e];
            if ((u & 0x7F80u) == 0x7F80u) u &= 0xffff0000u;
            if ((u & 0x7F800000u) == 0x7F800000u) u &= 0x0000ffffu;
            if (u != d[e]) {
                d[e] = u;
                odd = true;
            }
        }
    }
    return odd;
}
template <int HD>
__device__ __forceinline__ bool scrub_tile(unsigned char* tile, int first, int w, int lane) {
    constexpr int CH = HD / 8, RP = 32 / CH;
    const int c = lane % CH;
    const unsigned char* src = tile + (c >> 3) * 16384;
    uint32_t any = 0;
#pragma unroll 4
    for (int i = 0; i < 32 / RP; ++i) {
        const uint4 x = *reinterpret_cast<const uint4*>(src + sw128_offset(w * 32 + i * RP + lane / CH, c & 7));
        any |= (x.x & 0x7F807F80u) + 0x00800080u;
        any |= (x.y & 0x7F807F80u) + 0x00800080u;
        any |= (x.z & 0x7F807F80u) + 0x00800080u;
        any |= (x.w & 0x7F807F80u) + 0x00800080u;
    }
    return (any & 0x80008000u) != 0 && repair_tile<HD>(tile, first, w, lane);
}

// Four e4m3 numbers to bfloat16, times 2^-120: their 7 magnitude bits are moved to where
// bfloat16 keeps the low 4 exponent and high 3 fraction bits (subnormals to subnormals). Exact;
// the NaN codes come out as 480 and are looked for by the caller.
__device__ __forceinline__ void e4m3x4_to_bf16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    const uint32_t a = __byte_perm(w, 0, 0x1404), b = __byte_perm(w, 0, 0x3424);
    lo = ((a >> 4) & 0x07F007F0u) | (a & 0x80008000u);
    hi = ((b >> 4) & 0x07F007F0u) | (b & 0x80008000u);
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// What a row's numbers (times 2^-120) are multiplied by, as packed bfloat16: its scale 2^c times
// 2^120, in two factors (the second is 1 up to c = 7), so that neither overflows.
__device__ __forceinline__ uint2 scale_factors(float scale) {
    const int e = (int)(__float_as_uint(scale) >> 23) - 127 + 120, e1 = min(max(e, 0), 127), e2 = min(e - e1, 127);
    const uint32_t f1 = (uint32_t)(e1 + 127) << 7, f2 = (uint32_t)(max(e2, 0) + 127) << 7;
    return make_uint2(f1 | f1 << 16, f2 | f2 << 16);
}

// A lane's 16 numbers of a row, as two 16-byte chunks of a bfloat16 tile. Lanes of a row's second 64
// columns take their two halves in the other order, so that eight lanes store into different banks.
__device__ __forceinline__ void raw_words(const unsigned char* src, int c, uint32_t (&w)[4]) {
    const uint4 u = *reinterpret_cast<const uint4*>(src);
    const bool swap = c >> 2;
    w[0] = swap ? u.z : u.x;
    w[1] = swap ? u.w : u.y;
    w[2] = swap ? u.x : u.z;
    w[3] = swap ? u.y : u.w;
}
template <int HD>
__device__ __forceinline__ void store_converted(unsigned char* dst, int row, int c, const uint32_t (&o)[8]) {
    unsigned char* base = dst + (c >> 2) * 16384;
    const int swap = c >> 2, c0 = 2 * (c & 3) + swap, c1 = 2 * (c & 3) + 1 - swap;
    *reinterpret_cast<uint4*>(base + sw128_offset(row, c0)) = make_uint4(o[0], o[1], o[2], o[3]);
    *reinterpret_cast<uint4*>(base + sw128_offset(row, c1)) = make_uint4(o[4], o[5], o[6], o[7]);
}

// The warp's rows of a tile once more, with what convert_tile's loop leaves out: the second factor
// of scales above 2^7, NaN codes (to NaN, or in rows from `first` on to zero: returns whether there
// were any).
template <int HD>
__device__ __noinline__ bool convert_rare(const unsigned char* raw, uint2 mine, int first, unsigned char* dst, int w, int lane) {
    constexpr int CH = HD / 16, RP = 32 / CH;
    const int c = lane % CH;
    bool odd = false;
#pragma unroll 1
    for (int i = 0; i < 32 / RP; ++i) {
        const int r = i * RP + lane / CH, row = w * 32 + r;
        const uint32_t f1 = __shfl_sync(0xffffffffu, mine.x, r), f2 = __shfl_sync(0xffffffffu, mine.y, r);
        uint32_t in[4], o[8];
        raw_words(raw + row * HD + c * 16, c, in);
#pragma unroll
        for (int e = 0; e < 4; ++e) e4m3x4_to_bf16(in[e], o[2 * e], o[2 * e + 1]);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = mul_bf16x2(mul_bf16x2(o[e], f1), f2);
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (f1 != 0 && (in[e / 4] >> (8 * (e & 3)) & 0x7Fu) == 0x7Fu) {
                const uint32_t m = e & 1 ? 0xFFFF0000u : 0x0000FFFFu;
                o[e / 2] = (o[e / 2] & ~m) | (row >= first ? 0u : 0x7FC07FC0u & m);
                odd |= row >= first;
            }
        store_converted<HD>(dst, row, c, o);
    }
    return odd;
}

// One value tile of e4m3 rows, converted: raw [128][HD] bytes to the bfloat16 values they stand for
// (number * scale, exact); rows without a cache row become zero (their factor is zero). The loop
// has no branches; what it leaves out is looked for along the way and rarely found (convert_rare).
template <int HD>
__device__ __forceinline__ bool convert_tile(const unsigned char* raw, bool has_row, float scale, int first,
                                             unsigned char* dst, int w, int lane) {
    constexpr int CH = HD / 16, RP = 32 / CH;
    const int c = lane % CH;
    const uint2 mine = has_row ? scale_factors(scale) : make_uint2(0, 0x3F803F80u);
    const unsigned char* src = raw + (w * 32 + lane / CH) * HD + c * 16;
    uint32_t nan = 0;
#pragma unroll 1
    for (int i = 0; i < 32 / RP; ++i) {
        const int r = i * RP + lane / CH;
        const uint32_t f1 = __shfl_sync(0xffffffffu, mine.x, r);
        uint32_t in[4], o[8];
        raw_words(src + i * RP * HD, c, in);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            nan |= (in[e] & 0x7F7F7F7Fu) + 0x01010101u;
            e4m3x4_to_bf16(in[e], o[2 * e], o[2 * e + 1]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = mul_bf16x2(o[e], f1);
        store_converted<HD>(dst, w * 32 + r, c, o);
    }
    if (!__any_sync(0xffffffffu, (nan & 0x80808080u) != 0 || mine.y != 0x3F803F80u)) return false;
    return convert_rare<HD>(raw, mine, first, dst, w, lane);
}

// TMEM columns, not waited for; then the wait, which the values pass through
__device__ __forceinline__ void tc_ld16_start(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tc_ld16_wait(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :
                 : "memory");
}
__device__ __forceinline__ void tc_ld32_start(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tc_ld32_wait(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                   "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                   "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :
                 : "memory");
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

__device__ __forceinline__ float max32(const uint32_t* x) {
    float mx = __uint_as_float(x[0]), my = __uint_as_float(x[1]);
#pragma unroll
    for (int e = 2; e < 30; e += 4) {
        mx = max3(mx, __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
        my = max3(my, __uint_as_float(x[e + 2]), __uint_as_float(x[e + 3]));
    }
    mx = max3(mx, __uint_as_float(x[30]), __uint_as_float(x[31]));
    return fmaxf(mx, my);
}

// The rows of a warp move to references grown by log2(1 / f): the np packed columns of probabilities
// written so far at ts and the no columns of O at `to` times f. (Rare, hence a call.) TMEM loads are
// not ordered behind stores without a wait, and both may just have been stored: the probabilities by
// the softmax's last step, and everything by a rescaling one step earlier.
__device__ __noinline__ void rescale_row(uint32_t ts, int np, uint32_t to, int no, float f) {
    uint32_t u[16];
    tc_wait_st();
#pragma unroll 1
    for (int k = 0; k < np; k += 16) {
        tc_ld16_start(ts + k, u);
        tc_ld16_wait(u);
#pragma unroll
        for (int e = 0; e < 16; ++e)
            u[e] = pack_bf16(__uint_as_float(u[e] << 16) * f, __uint_as_float(u[e] & 0xFFFF0000u) * f);
        tc_st16(ts + k, u);
    }
#pragma unroll 1
    for (int k = 0; k < no; k += 16) {
        tc_ld16_start(to + k, u);
        tc_ld16_wait(u);
#pragma unroll
        for (int e = 0; e < 16; ++e) u[e] = __float_as_uint(__uint_as_float(u[e]) * f);
        tc_st16(to + k, u);
    }
}

// One row's softmax of a tile, in one pass over its 128 scores x at TMEM columns ts: 2^(scale2 x - m)
// as packed bfloat16 over the first 64 columns (32 scores become 16 columns, always behind what is
// still to be read), their float32 sum added to `sum`. m is the row's reference, its maximum rounded
// up to a whole number; when some row of the warp has outgrown it by more than 2^12, the warp moves to
// new references on the spot. They differ by whole numbers, so what has been written is scaled by a
// power of two and not rounded again.
// Bound by latency: the next 32 scores load under the exponentials of these (512 of a tile's 1300
// clocks), their maximum follows. A loop with a short body: the CTA's roles share the instruction caches, and
// unrolled rows made every one of them wait for fetches.
// With e4m3 keys (Q8) the scores still lack their keys' scales, ks (shared memory).
template <int HD, bool Q8>
__device__ __forceinline__ void softmax_row(uint32_t ts, uint32_t to, float scale2, bool first, const float* ks, float& m,
                                            float& sum) {
    const uint64_t sc = pair_f32(__float_as_uint(scale2), __float_as_uint(scale2));
    uint32_t x[32], y[32];
    uint64_t z[2] = {0, 0};
    auto scale32 = [&](uint32_t* v, int c) {
        if constexpr (Q8) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
                const float4 f = *reinterpret_cast<const float4*>(ks + c + e);
                const uint64_t a = mul_x2(pair_f32(v[e], v[e + 1]), pair_f32(__float_as_uint(f.x), __float_as_uint(f.y)));
                const uint64_t b = mul_x2(pair_f32(v[e + 2], v[e + 3]), pair_f32(__float_as_uint(f.z), __float_as_uint(f.w)));
                v[e] = (uint32_t)a;
                v[e + 1] = (uint32_t)(a >> 32);
                v[e + 2] = (uint32_t)b;
                v[e + 3] = (uint32_t)(b >> 32);
            }
        }
    };
    tc_ld32_start(ts, x);
    tc_ld32_wait(x);
    scale32(x, 0);
    float mx = max32(x) * scale2;
#pragma unroll 1
    for (int c = 0; c < kTcTile; c += 32) {
        if (__any_sync(0xffffffffu, mx > m + kRescale)) {
            const float mn = fmaxf(m, ceilf(mx)), d = mn == -INFINITY ? 0.f : m - mn;  // (whole, or -inf)
            const float f = d < -126.f ? 0.f : __uint_as_float((uint32_t)(127 + (int)d) << 23);
            const uint64_t ff = pair_f32(__float_as_uint(f), __float_as_uint(f));
            z[0] = fma_x2(z[0], ff, 0);
            z[1] = fma_x2(z[1], ff, 0);
            sum *= f;
            m = mn;
            rescale_row(ts, c / 2, to, first ? 0 : HD, f);
        }
        const float shift = m == -INFINITY ? 0.f : -m;
        const uint64_t sh = pair_f32(__float_as_uint(shift), __float_as_uint(shift));
        uint32_t pk[16];
        auto exps = [&](int e0) {
#pragma unroll
            for (int e = e0; e < e0 + 16; e += 2) {
                const uint64_t v = fma_x2(pair_f32(x[e], x[e + 1]), sc, sh);
                const float p0 = ex2_approx(__uint_as_float((uint32_t)v)), p1 = ex2_approx(__uint_as_float((uint32_t)(v >> 32)));
                z[(e >> 1) & 1] = add_x2(z[(e >> 1) & 1], pair_f32(__float_as_uint(p0), __float_as_uint(p1)));
                pk[e / 2] = pack_bf16(p0, p1);
            }
        };
        // (past the last column the first ones are loaded again, and not used)
        tc_ld32_start(ts + (c + 32) % kTcTile, y);
        exps(0);
        tc_ld32_wait(y);
        exps(16);
        scale32(y, (c + 32) % kTcTile);
        mx = max32(y) * scale2;
        tc_st16(ts + c / 2, pk);
#pragma unroll
        for (int e = 0; e < 32; ++e) x[e] = y[e];
    }
    const uint64_t zz = add_x2(z[0], z[1]);
    sum += __uint_as_float((uint32_t)zz) + __uint_as_float((uint32_t)(zz >> 32));
}

// Ring positions of a segment's tiles. They are loaded in the order of their first use:
// K0 K1 V0 K2 V1 ... K(n-1) V(n-2) V(n-1).
__device__ __forceinline__ int pos_k(int t) { return t == 0 ? 0 : 2 * t - 1; }
__device__ __forceinline__ int pos_v(int t, int n) { return t < n - 1 ? 2 * t + 2 : 2 * n - 1; }
__device__ __forceinline__ bool tile_is_value(int l, int n) { return l == 2 * n - 1 || (l > 0 && !(l & 1)); }
__device__ __forceinline__ int tile_number(int l, int n) {
    return l == 0 ? 0 : l == 2 * n - 1 ? n - 1 : l & 1 ? (l + 1) / 2 : (l - 2) / 2;
}

// Whether 16 bytes of a cache row hold an infinity or NaN; element e of them: 0 finite, 1 NaN, 2 +inf, 3 -inf
template <bool Q8>
__device__ __forceinline__ bool odd_chunk(uint4 u) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    uint32_t any = 0;  // (a NaN code's low bits, or an exponent of ones, carry into the bit above)
#pragma unroll
    for (int k = 0; k < 4; ++k) any |= Q8 ? (w[k] & 0x7F7F7F7Fu) + 0x01010101u : ((w[k] & 0x7F807F80u) + 0x00800080u);
    return (any & 0x80808080u) != 0 && (Q8 || (any & 0x80008000u) != 0);
}
template <bool Q8>
__device__ __forceinline__ int odd_kind(uint4 u, int e) {
    const int k = Q8 ? e >> 2 : e >> 1;
    const uint32_t w = k == 0 ? u.x : k == 1 ? u.y : k == 2 ? u.z : u.w;
    if (Q8) return (w >> (8 * (e & 3)) & 0x7Fu) == 0x7Fu ? 1 : 0;
    const uint32_t x = w >> (16 * (e & 1)) & 0xFFFFu;
    return (x & 0x7F80u) != 0x7F80u ? 0 : x & 0x7Fu ? 1 : x & 0x8000u ? 3 : 2;
}

// For a row that sees non-finite value elements of nodes (which the loaders set to zero): they are
// added to the result in their columns, which become that infinity, or NaN where a NaN, infinities
// of both signs or a probability of exactly zero (a score of -inf) are among them. What they are
// multiplied by does not matter otherwise, so the values are only looked through, each once a row
// and until all columns are NaN: this takes about as long as the row's nodes have value bytes, and a
// prompt whose values are all NaN keeps no other role waiting. The result may hold an infinity or
// NaN of the prefix already. dst: the row's place in the output (bfloat16) or the partial results
// (float32), where this thread has just written the rest.
template <int HD, bool Q8>
__device__ __noinline__ void put_odd_columns(const TreeAttnArgs& a, const Segment& g, int node, int head, void* dst, int e0, int e1) {
    constexpr int E = Q8 ? 16 : 8, CH = HD / E;          // elements of 16 bytes, chunks of a row
    constexpr int AT = CH / 2 < 4 ? CH / 2 : 4;  // chunks loaded at a time (of half a row or all of it)
    const bf16_t* q = (const bf16_t*)a.q.p + g.b * a.q.batch + (int64_t)node * a.q.token + (int64_t)head * a.q.head;
    unsigned long long kind[3][2] = {{0, 0}, {0, 0}, {0, 0}};  // columns with a NaN, a +inf, a -inf
    // a score of -inf takes an infinity in the key or the query (e4m3 makes NaN of either)
    int odd_q = -1;
    auto minus_inf = [&](int64_t row) -> bool {
        if (Q8) return false;
        const uint4* k = reinterpret_cast<const uint4*>(a.cache.k) + row * CH;
        bool odd = false;
#pragma unroll 4
        for (int c = 0; c < CH; ++c) odd |= odd_chunk<Q8>(k[c]);
        if (odd_q < 0) {
            odd_q = 0;
#pragma unroll 1
            for (int e = 0; e < HD; ++e) odd_q |= !finite_f32(Storage<bf16_t>::load(q, e));
        }
        if (!odd && !odd_q) return false;
        float dot = 0.f;
#pragma unroll 1
        for (int e = 0; e < HD; ++e) dot = fmaf(Storage<bf16_t>::load(q, e), Storage<bf16_t>::load((const bf16_t*)k, e), dot);
        return dot == -INFINITY;
    };
#pragma unroll 1
    for (int tile = max(g.s.P / kTcTile, g.t0); tile < g.t1; ++tile) {
        const int s0 = tile * kTcTile;
        const ulonglong2 see = seen_bits(a, g, node, s0);
#pragma unroll 1
        for (int r = max(g.s.P - s0, 0); r < min(g.end - s0, kTcTile); ++r) {
            if (!((r < 64 ? see.x >> r : see.y >> (r - 64)) & 1ull)) continue;
            const RowInfo x = row_info<Q8>(a, g, tile, r);
            if (x.row < 0) continue;
            const uint4* v = reinterpret_cast<const uint4*>(a.cache.v) + x.row * CH;
            int none = -1;  // the slot's probability is zero (-1: not looked at)
#pragma unroll 1
            for (int c = e0 / E; c < e1 / E; c += AT) {
                uint4 u[AT];
                bool odd = false;
#pragma unroll
                for (int k = 0; k < AT; ++k) u[k] = v[c + k];
#pragma unroll
                for (int k = 0; k < AT; ++k) odd |= odd_chunk<Q8>(u[k]);
                if (!odd) continue;
                if (none < 0) none = minus_inf(x.row);
#pragma unroll
                for (int i = 0; i < AT * E; ++i) {
                    const int k = odd_kind<Q8>(u[i / E], i % E), e = c * E + i;
                    if (k) kind[none ? 0 : k - 1][e >> 6] |= 1ull << (e & 63);
                }
            }
            if (__popcll(kind[0][0]) + __popcll(kind[0][1]) == e1 - e0) {
                tile = g.t1;
                break;
            }
        }
    }
#pragma unroll 1
    for (int e = e0; e < e1; ++e) {
        auto has = [&](int k) { return (kind[k][e >> 6] >> (e & 63) & 1ull) != 0; };
        const bool nan = has(0), pos = has(1), neg = has(2);
        if (!nan && !pos && !neg) continue;
        const float t = nan || (pos && neg) ? __uint_as_float(0x7FC00000u) : pos ? INFINITY : -INFINITY;
        if (g.whole) store_one((bf16_t*)dst + e, Storage<bf16_t>::load((const bf16_t*)dst, e) + t);
        else ((float*)dst)[e / 4 * (4 * kAttnItemRows) + e % 4] += t;
    }
}

// A query row, for the e4m3 product with keys as they are: q = 2^c (hi + lo), hi the e4m3 rounding
// of q / 2^c with the smallest c that fits the row's largest magnitude under 448, lo that of the
// rest. A bfloat16 number's 8 significant bits are two times e4m3's 4, so the split is exact for
// elements from 2^c / 4 on (2^-9 of the row's largest is always that); smaller ones end at e4m3's
// last place and are off by up to 2^(c - 10), 2^-17 of the largest, where bfloat16 held more. It costs
// the tensor cores nothing: two products at twice the rate. (Keys converted to bfloat16 would meet
// queries as they are: 423 us where this took 390, 81 nodes over 131k slots.) In place: the 64 bytes of elements 32 k .. become their 32 hi
// and 32 lo bytes. Returns 2^c.
template <int HD>
__device__ __forceinline__ float split_query_row(unsigned char* block, int row) {
    auto chunk = [&](int c) { return reinterpret_cast<uint4*>(block + (c >> 3) * 16384 + sw128_offset(row, c & 7)); };
    float m = 0.f;
#pragma unroll 1
    for (int c = 0; c < HD / 8; ++c) {
        float x[8];
        Vec16<bf16_t>::widen(*chunk(c), x);
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_f32(x[e]) ? fabsf(x[e]) : 0.f);
    }
    const uint32_t u = __float_as_uint(m);
    const int c2 = max((int)(u >> 23) - 135 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0), -100);
    const float inv = __uint_as_float((uint32_t)(127 - c2) << 23);
#pragma unroll 1
    for (int k = 0; k < HD / 32; ++k) {
        uint4 v[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = *chunk(4 * k + c);
        uint32_t hi[8], lo[8];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float x[8];
            Vec16<bf16_t>::widen(v[c], x);
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                uint32_t h[2], l[2];
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const float a = x[e + 2 * z], b = x[e + 2 * z + 1];
                    const float y0 = finite_f32(a) ? a * inv : __uint_as_float(0x7FC00000u);
                    const float y1 = finite_f32(b) ? b * inv : __uint_as_float(0x7FC00000u);
                    h[z] = f32x2_to_e4m3(y0, y1);
                    const float2 f = e4m3x2_to_f32(h[z]);
                    l[z] = f32x2_to_e4m3(y0 - f.x, y1 - f.y);
                }
                hi[2 * c + e / 4] = h[0] | h[1] << 16;
                lo[2 * c + e / 4] = l[0] | l[1] << 16;
            }
        }
        *chunk(4 * k) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *chunk(4 * k + 1) = make_uint4(hi[4], hi[5], hi[6], hi[7]);
        *chunk(4 * k + 2) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        *chunk(4 * k + 3) = make_uint4(lo[4], lo[5], lo[6], lo[7]);
    }
    return __uint_as_float((uint32_t)(127 + c2) << 23);
}

// Whether a tile of a bfloat16 cache comes by TMA: all do where a box holds 32 rows or more; of
// smaller pages' the loaders bring the values, except those to look through.
constexpr int kWideBox = 32;
__device__ __forceinline__ bool by_tma(const TreeAttnArgs& a, const Segment& g, int tt, bool val) {
    return a.box_rows >= kWideBox || (a.box_rows > 0 && (!val || (g.t0 + tt + 1) * kTcTile > g.s.P));
}

// A position in the ring of tiles: slot and phase, moved on by small steps without division.
template <int S>
struct RingPos {
    int slot = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void skip(int d) {
        slot += d;
#pragma unroll
        for (int k = 0; k < 2; ++k)  // (d <= 2 S)
            if (slot >= S) {
                slot -= S;
                phase ^= 1u;
            }
    }
    __device__ __forceinline__ void skip_long(int d) {
        phase ^= (uint32_t)((slot + d) / S) & 1u;
        slot = (slot + d) % S;
    }
};

// ---- the kernel -----------------------------------------------------------------------------------
template <int HD, bool Q8, int MT>
__global__ void __launch_bounds__(TcShape<HD, Q8, MT>::kThreads, 1)
    tree_attn_tc_kernel(const __grid_constant__ TreeAttnArgs a, const __grid_constant__ CUtensorMap kmap,
                        const __grid_constant__ CUtensorMap vmap, const __grid_constant__ CUtensorMap qmap) {
    using SH = TcShape<HD, Q8, MT>;
    constexpr int S = SH::kSlots, KS = Q8 ? SH::kKeySlots : 1, RS = Q8 ? SH::kRawSlots : 1, TB = SH::kTileBytes;
    extern __shared__ __align__(1024) unsigned char qbuf[];
    unsigned char* ring = qbuf + MT * TB;
    unsigned char* keyring = ring + S * TB;  // (e4m3)
    unsigned char* rawring = keyring + SH::kKeySlots * SH::kRawBytes;
    float* key_scales = (float*)(rawring + SH::kRawSlots * SH::kRawBytes);
    float* query_scales = key_scales + kTcScales * kTcTile;
    TcState& st = *reinterpret_cast<TcState*>(qbuf + SH::kData);
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    griddep_launch_dependents();
    // what takes long and needs nothing goes first: the schedule, and the tensor maps' descriptors
    PlanArgs pa = plan_args(a);
    bool bad = false;
    SegmentWalk<TcPlan<Q8>> walk;
    // (nothing to join, until the planner has come to its end: a CTA that gives up leaves no old note)
    if (warp == 14 && lane == 0) a.split[blockIdx.x] = SplitDesc{0, 0, 0, 0, -1, 0, {0, 0}};
    if (warp == 14) walk.init(pa, blockIdx.x, gridDim.x, &bad);
    if (warp == 15 && lane < 3) {
        const CUtensorMap* map = lane == 0 ? &kmap : lane == 1 ? &vmap : &qmap;
        if (lane == 2 ? a.q_tma : a.box_rows > 0 && (lane == 0 || !Q8))
            asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
    }
    if (smem_u32(qbuf) & 1023u) {  // (dynamic memory alone starts on a 1024-byte boundary)
        if (t == 0) atomicOr(a.status, ST_DEVICE);
        return;
    }

    if (t == 0) {
        for (int i = 0; i < S; ++i) {
            mbar_init(&st.full[i], 128);
            mbar_init(&st.landed[i], 1);
            mbar_init(&st.empty[i], MT);  // (a tile that one stream alone used is released twice by it)
        }
        for (int i = 0; i < KS; ++i) {
            mbar_init(&st.kfull[i], 129);  // the loaders (scales) and the TMA warp (keys)
            mbar_init(&st.kempty[i], MT);
        }
        for (int i = 0; i < RS; ++i) {
            mbar_init(&st.rawfull[i], 1);
            mbar_init(&st.rawempty[i], 128);
        }
        for (int i = 0; i < kTcSegs; ++i) {
            mbar_init(&st.segfull[i], 1);
            mbar_init(&st.segempty[i], SH::kReaders);
        }
        mbar_init(&st.qfull, 256);
        mbar_init(&st.qempty, 2);  // both streams' score products
        mbar_init(&st.qready, 8);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&st.sfull[i], 1);
            mbar_init(&st.pfull[i], 4);
            mbar_init(&st.drain[i], 1);
            mbar_init(&st.turn[i], 1);
            mbar_init(&st.odone[i], 1);
        }
        mbar_init(&st.ofree, 8);
        mbar_init(&st.mlfull, 8);
        mbar_init(&st.mlfree, 8);
        st.abort = 0;
        for (int i = 0; i < 8; ++i) st.odd[i] = 0;
        mbar_fence_init();
    }
    if (warp == 12) tc_alloc(&st.tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = st.tmem;
    // Whole warps wait together and agree on the outcome: a warp of which some lanes gave up would not
    // meet again at the warp-wide instructions that follow.
    auto wait = [&](uint64_t* bar, uint32_t parity, int tiles = 0) {
        return __all_sync(0xffffffffu, mbar_try_wait(bar, parity & 1u)) ||
               tc_wait_slow(bar, parity & 1u, a.status, &st.abort, kWaitBudgetNs + tiles * kTileBudgetNs);
    };
    // the next planned segment; false at the end (or after a failed wait)
    uint32_t seg = 0;  // segments taken
    auto next = [&](Segment& g) -> bool {
        const int k = seg % kTcSegs;
        if (!wait(&st.segfull[k], seg / kTcSegs)) return false;
        g = st.seg[k];
        __syncwarp();
        if (lane == 0) mbar_arrive(&st.segempty[k]);
        ++seg;
        return g.weight != 0;
    };
    Segment g;
    bool ok = true;
    // What a role that issues bulk copies has issued, for the wait at the end: where waits have failed,
    // nobody else may have waited for the last of them.
    uint32_t sent = 0;

    if (Q8 && warp >= 8 && warp < 12) {  // ---- loaders of an e4m3 cache: key scales, value conversion
        const int w = warp - 8, r = w * 32 + lane;  // the lane's row of every tile
        RingPos<S> pos;
        RingPos<KS> kpos;
        RingPos<RS> rpos;
        bool reuse = false, kreuse = false;  // the rings have been filled once
        uint32_t tiles = 0;  // key tiles so far
        while (ok && next(g)) {
            const int nt = g.t1 - g.t0;
            // the row's place and scales in tiles tt and tt + 1; the next tile's are fetched a tile ahead
            RowInfo x1 = row_info<Q8>(a, g, g.t0, r);
            float vs = 0.f;
            bool has = false;
#pragma unroll 1
            for (int tt = -1; tt < nt; ++tt) {  // K0 (K1 V0) (K2 V1) ...
                const float vs1 = x1.vs;
                const bool has1 = x1.row >= 0, ok1 = has1 && (!x1.node || valid_scale(vs1));
                if (tt + 1 < nt) {  // the rows' scales; the rows themselves where TMA cannot fetch them
                    if (kreuse && !(ok = wait(&st.kempty[kpos.slot], kpos.phase ^ 1u))) break;
                    key_scales[(tiles++ % kTcScales) * kTcTile + r] = has1 && (!x1.node || valid_scale(x1.ks)) ? x1.ks : 1.f;
                    if (a.box_rows > 0) {
                        mbar_arrive(&st.kfull[kpos.slot]);
                    } else {
                        load_key_tile<HD>(a.cache.k, x1, keyring + kpos.slot * SH::kRawBytes, w, lane);
                        cp_async_arrive(&st.kfull[kpos.slot]);
                    }
                    kpos.skip(1);
                    kreuse |= kpos.slot == 0;
                    x1 = row_info<Q8>(a, g, g.t0 + tt + 2, r);
                }
                if (tt >= 0) {
                    if (!(ok = wait(&st.rawfull[rpos.slot], rpos.phase))) break;
                    if (reuse && !(ok = wait(&st.empty[pos.slot], pos.phase ^ 1u))) break;
                    // (the MMA warp's proxy fence orders the tile's writes before the product's reads)
                    if (convert_tile<HD>(rawring + rpos.slot * SH::kRawBytes, has, vs, g.s.P - (g.t0 + tt) * kTcTile,
                                         ring + pos.slot * TB, w, lane))
                        st.odd[(seg - 1) & 7] = 1;
                    mbar_arrive(&st.rawempty[rpos.slot]);
                    mbar_arrive(&st.full[pos.slot]);
                    rpos.skip(1);
                    pos.skip(1);
                    reuse |= pos.slot == 0;
                }
                vs = vs1;
                has = ok1;
            }
        }
        cp_async_wait_all();
    } else if (warp >= 8 && warp < 12) {  // ---- loaders of a bfloat16 cache
        const int w = warp - 8;
        RingPos<S> pos;
        bool reuse = false;       // the ring has been filled once
        uint32_t landed = 0;      // by slot: the phase of landed[] that comes next
        while (ok && next(g)) {
            const int nt = g.t1 - g.t0;
#pragma unroll 1
            for (int l = 0; l < 2 * nt; ++l) {  // K0 K1 V0 K2 V1 ...
                const bool val = tile_is_value(l, nt);
                const int tt = tile_number(l, nt);
                unsigned char* dst = ring + pos.slot * TB;
                uint64_t* full = &st.full[pos.slot];
                const int first = g.s.P - (g.t0 + tt) * kTcTile;  // first row of the tile that is a node's
                // (where the loaders fill slots, every slot's release is waited for: a barrier's phase is one
                // bit, and a role that skipped one could take an older release for the one it needs)
                if (a.box_rows < kWideBox && reuse && !(ok = wait(&st.empty[pos.slot], pos.phase ^ 1u))) break;
                if (by_tma(a, g, tt, val)) {  // what TMA brings is looked through where it may hold what nobody sees
                    if (val && first < kTcTile) {
                        if (!(ok = wait(&st.landed[pos.slot], landed >> pos.slot))) break;
                        landed ^= 1u << pos.slot;
                        if (scrub_tile<HD>(dst, first, w, lane)) {
                            st.odd[(seg - 1) & 7] = 1;
                            fence_async_proxy();
                        }
                        mbar_arrive(full);
                    }
                } else {
                    const RowInfo x = row_info<Q8>(a, g, g.t0 + tt, w * 32 + lane);
                    load_tile<HD>(val ? a.cache.v : a.cache.k, x, dst, w, lane);
                    if (val && first < kTcTile) {
                        cp_async_wait_all();
                        if (scrub_tile<HD>(dst, first, w, lane)) st.odd[(seg - 1) & 7] = 1;
                        fence_async_proxy();
                        mbar_arrive(full);
                    } else {
                        // (the copies' writes are ordered before the MMA's reads by the MMA warp's
                        // proxy fence: a fence here would wait for the copies)
                        cp_async_arrive(full);
                    }
                }
                pos.skip(1);
                reuse |= pos.slot == 0;
            }
        }
        cp_async_wait_all();
    } else if (warp == 12 || warp == 13) {  // ---- MMA issuers, one thread per stream
        const int gs = warp - 12;
        const uint32_t id_qk = Q8 ? idesc_e4m3_f32(128, kTcTile) : idesc_bf16_f32(128, kTcTile);
        const uint32_t id_pv = idesc_bf16_f32(128, HD) | (1u << 16);  // B is MN-major
        const uint32_t ts = tmem + gs * 128, to = tmem + 256 + gs * 128;
        const uint64_t ring_d = sw128_desc(smem_u32(ring)), ring_mn = sw128_desc_mn(smem_u32(ring), 16384);
        // The streams take turns: a stream's P V and next Q K^T are issued together and run while the
        // other's softmax does. (Issued side by side, both streams' products end together and then
        // both softmaxes compete.) The warp runs as one, and one lane issues.
        const uint64_t key_d = key_desc<HD>(smem_u32(keyring));
        // keys and values: positions in one ring, or (e4m3) in a ring each
        constexpr int KR = Q8 ? KS : S;
        uint64_t* const kfull = Q8 ? st.kfull : st.full;
        uint64_t* const kempty = Q8 ? st.kempty : st.empty;
        RingPos<S> base;
        RingPos<KR> kbase;
        uint32_t np = 0, turn = 0;
        while (ok && next(g)) {
            const int nt = g.t1 - g.t0;
            const bool pair = g.weight == 2;
            const int step = pair ? 1 : 2, first = pair ? 0 : gs;
            const uint64_t qd = sw128_desc(smem_u32(qbuf + (pair ? gs * TB : 0)));
            const bool twice = MT == 2 && !pair;
            RingPos<KR> kp = kbase;
            RingPos<S> vp = base;
            kp.skip(Q8 ? first : pos_k(first));
            vp.skip(Q8 ? first : pos_v(first, nt));
            if (first < nt) ok = wait(Q8 ? &st.qready : &st.qfull, seg - 1);
            bool qdone = false;
            // (both streams make the same number of rounds, the last of stream 1 may be empty)
#pragma unroll 1
            for (int t0 = -step; t0 < nt && ok; t0 += step) {  // O += P V of tile tt, S = Q K^T of the next
                const int tt = t0 + first;
                const bool pv = t0 >= 0 && tt < nt, qk = tt + step < nt;
                // the tiles first (K only if it is there already), with the proxy fence that they need; the
                // probabilities, which are what is late as a rule, and the stream's turn after it
                if (pv) ok = ok && wait(&st.full[vp.slot], vp.phase);
                bool kthere = qk && mbar_try_wait(&kfull[kp.slot], kp.phase);
                kthere = __all_sync(0xffffffffu, kthere);
                fence_async_proxy();
                if (pv) {
                    if (t0 == 0 && seg > 1) ok = ok && wait(&st.ofree, seg - 2);
                    ok = ok && wait(&st.pfull[gs], np);
                    ++np;
                }
                if (gs == 1 || turn > 0) ok = ok && wait(&st.turn[gs], gs == 1 ? turn : turn - 1);
                ++turn;
                if (!__all_sync(0xffffffffu, ok)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const bool leader = elect_one();
                if (pv && leader) {
                    const uint64_t vd = ring_mn + (uint32_t)(vp.slot * (TB / 16));
#pragma unroll
                    for (int k = 0; k < kTcTile / 16; ++k)
                        tc_mma_ts(to, ts + k * 8, vd + k * 128, id_pv, t0 > 0 || k ? 1u : 0u);
                }
                if (qk && !kthere) {
                    ok = __all_sync(0xffffffffu, wait(&kfull[kp.slot], kp.phase));
                    if (!ok) break;
                    fence_async_proxy();
                    tc_fence_after();
                }
                if (leader) {
                    if (qk && Q8) {
                        const uint64_t kd = key_d + (uint32_t)(kp.slot * (SH::kRawBytes / 16));
#pragma unroll
                        for (int k = 0; k < HD / 16; ++k)  // 32 elements' hi, then their lo part, with the same keys
                            tc_mma_e4m3(ts, qd + (k >> 2) * 1024 + 2 * (k & 3), kd + 2 * (k >> 1), id_qk, k ? 1u : 0u);
                        tc_commit(&st.sfull[gs]);
                    } else if (qk) {
                        const uint64_t kd = ring_d + (uint32_t)(kp.slot * (TB / 16));
#pragma unroll
                        for (int k = 0; k < HD / 16; ++k)  // 32 bytes a step, 16384 to the next 64 columns
                            tc_mma(ts, qd + (k >> 2) * 1024 + 2 * (k & 3), kd + (k >> 2) * 1024 + 2 * (k & 3), id_qk, k ? 1u : 0u);
                        tc_commit(&st.sfull[gs]);
                    }
                    mbar_arrive(&st.turn[gs ^ 1]);
                    if (qk) {
                        tc_commit(&kempty[kp.slot]);
                        if (twice) tc_commit(&kempty[kp.slot]);
                        if (tt + 2 * step >= nt) tc_commit(&st.qempty);
                    }
                    if (pv) {
                        tc_commit(&st.empty[vp.slot]);
                        if (twice) tc_commit(&st.empty[vp.slot]);
                    }
                }
                __syncwarp();
                if (pv) vp.skip(Q8 ? step : pos_v(min(tt + step, nt - 1), nt) - pos_v(tt, nt));
                if (qk) kp.skip(Q8 ? step : 2 * step - (tt + step == 0));
                qdone |= qk;
            }
            if (ok && elect_one()) {
                if (!qdone) tc_commit(&st.qempty);
                tc_commit(&st.odone[gs]);
            }
            __syncwarp();
            base.skip_long(Q8 ? nt : 2 * nt);
            kbase.skip_long(Q8 ? nt : 2 * nt);
        }
        // every MMA issued has finished reading shared memory and TMEM before the CTA ends
        if (elect_one()) tc_commit(&st.drain[gs]);
        __syncwarp();
        mbar_wait(&st.drain[gs], 0, a.status, 100000000LL);
    } else if (warp == 14) {  // ---- the plan
        if (bad && blockIdx.x == 0) atomicOr(a.status, ST_CAPACITY);
        // It alone waits for as long as a whole segment takes, which may have two million tiles.
        uint32_t n = 0;
        int longest = 0;  // tiles of a segment so far
        bool continues = false;
        for (; ok; ++n) {
            const bool more = walk.next(pa, g);
            continues |= more && !g.whole && g.slot == 0;
            if (!more && lane == 0) a.split[blockIdx.x] = walk.desc(pa, n > 0, g, continues);
            const int k = n % kTcSegs;
            if (n >= kTcSegs && !(ok = wait(&st.segempty[k], n / kTcSegs - 1, longest))) break;
            if (lane == 0) {
                if (!more) g.weight = 0;
                st.seg[k] = g;
                mbar_arrive(&st.segfull[k]);
            }
            __syncwarp();
            if (!more) break;
            const int before = longest;  // (of the segments that a wait here may last)
            longest = max(longest, g.t1 - g.t0);
            if (a.q_tma) {  // the queries, once the buffer's last ones are done with
                if (n > 0 && !(ok = wait(&st.qempty, n - 1, before))) break;
                if (lane == 0) {
                    mbar_arrive_expect_tx(&st.qfull, g.weight * TB);
                    mbar_arrive_n(&st.qfull, 255);  // in the place of the softmax warps' 256 arrivals
                    const int per = 128 / a.G;  // nodes of a block; its rows are their heads of this KV head
                    for (int b = 0; b < g.weight; ++b)
                        for (int half = 0; half < HD / 64; ++half)
                            tma_load_4d(smem_u32(qbuf) + b * TB + half * 16384, &qmap, half * 64, g.h * a.G,
                                        (2 * g.m + b) * per, g.b, &st.qfull);
                }
                __syncwarp();
            }
        }
        sent = a.q_tma ? n : 0;
    } else if (Q8 && warp == 15) {  // ---- an e4m3 cache's keys (TMA) and raw values (bulk copies)
        RingPos<KS> kpos;
        RingPos<RS> pos;
        bool kreuse = false;
        uint32_t i = 0, ktiles = 0;
        while (ok && next(g)) {
            const int nt = g.t1 - g.t0;
            const int br = a.box_rows > 0 ? a.box_rows : kTcTile, boxes = kTcTile / br;
#pragma unroll 1
            for (int l = 0; l < 2 * nt; ++l) {
                const int tt = tile_number(l, nt);
                const int s0 = (g.t0 + tt) * kTcTile, s1 = min(s0 + kTcTile, g.end);
                if (!tile_is_value(l, nt)) {
                    if (kreuse && !(ok = wait(&st.kempty[kpos.slot], kpos.phase ^ 1u))) break;
                    uint64_t* full = &st.kfull[kpos.slot];
                    if (a.box_rows > 0) {
                        if (lane == 0) mbar_arrive_expect_tx(full, SH::kRawBytes);
                        __syncwarp();
                        if (lane < boxes) {  // a box of rows a lane; boxes past the item's end read as zeros, or hidden rows
                            const int slot = s0 + lane * br;
                            int y = slot, z = g.b * a.Hkv + g.h;
                            if (a.cache.page_size) {
                                const int lp = slot / a.cache.page_size;
                                y = slot - lp * a.cache.page_size;
                                z = a.cache.n_pages * a.Hkv;  // past the pool
                                if (slot < g.end) {
                                    const int pg = a.cache.table[(int64_t)g.b * a.cache.max_pages + lp];
                                    if (pg >= 0 && pg < a.cache.n_pages) z = pg * a.Hkv + g.h;
                                    else atomicOr(a.status, ST_DEVICE);
                                }
                            }
                            tma_load_3d(smem_u32(keyring) + kpos.slot * SH::kRawBytes + lane * br * HD, &kmap, 0, y, z, full);
                        }
                    } else if (lane == 0) {
                        mbar_arrive(full);
                    }
                    ++ktiles;
                    kpos.skip(1);
                    kreuse |= kpos.slot == 0;
                    continue;
                }
                if (i >= (uint32_t)RS && !(ok = wait(&st.rawempty[pos.slot], pos.phase ^ 1u))) break;
                const int ps = a.cache.page_size ? a.cache.page_size : a.cache.max_seq;
                const int p0 = s0 / ps, np = (s1 - 1) / ps - p0 + 1;
                // a lane's runs of rows: pages p0 + lane, + 32, ...
                auto run = [&](int k, int& from, int& rows, int64_t& row) -> bool {
                    const int lo = max(s0, (p0 + k) * ps), hi = (int)min((int64_t)s1, (int64_t)(p0 + k + 1) * ps);
                    from = lo - s0;
                    rows = hi - lo;
                    if (!cache_row(a.cache, g.b, lo, row, a.status)) return false;
                    row += g.h * head_step(a.cache);
                    return true;
                };
                // the first round's runs stay at hand; more than 32 pages are looked up again
                int from = 0, rows = 0, bytes = 0;
                int64_t row = 0;
                const bool mine = lane < np && run(lane, from, rows, row);
                if (mine) bytes = rows * HD;
                int f2, r2;
                int64_t w2;
#pragma unroll 1
                for (int k = lane + 32; k < np; k += 32)
                    if (run(k, f2, r2, w2)) bytes += r2 * HD;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) bytes += __shfl_xor_sync(0xffffffffu, bytes, o);
                uint64_t* full = &st.rawfull[pos.slot];
                if (lane == 0) mbar_arrive_expect_tx(full, bytes);
                __syncwarp();
                unsigned char* dst = rawring + pos.slot * SH::kRawBytes;
                const char* src = (const char*)a.cache.v;
                if (mine) bulk_g2s(dst + from * HD, src + row * HD, rows * HD, full);
#pragma unroll 1
                for (int k = lane + 32; k < np; k += 32)
                    if (run(k, f2, r2, w2)) bulk_g2s(dst + f2 * HD, src + w2 * HD, r2 * HD, full);
                pos.skip(1);
                ++i;
            }
        }
        // leave with no copy in flight: the last tiles have landed
        for (uint32_t j = i > (uint32_t)RS ? i - RS : 0; j < i; ++j) mbar_wait(&st.rawfull[j % RS], (j / RS) & 1u, a.status);
        sent = a.box_rows > 0 ? ktiles : 0;
    } else if (!Q8 && warp == 15) {  // ---- a bfloat16 cache's tiles by TMA
        RingPos<S> pos;
        bool reuse = false;
        // (sent, by slot: used; from bit 8 its last use's phase; from bit 16: on landed[])
        uint32_t landed = 0;  // by slot: the phase of landed[] that comes next
        while (ok && a.box_rows > 0 && next(g)) {
            const int nt = g.t1 - g.t0;
            // a lane's box of every tile: rows box * br .. of the tile, columns half * 64 ..
            const int br = a.box_rows, boxes = kTcTile / br, box = lane % boxes, half = lane / boxes;
            // where tile t's box lies: its page's (or sequence's) place in the map; fetched a tile ahead
            auto place = [&](int t) -> int {
                if (!a.cache.page_size) return g.b * a.Hkv + g.h;
                const int slot = (g.t0 + t) * kTcTile + box * br, lp = slot / a.cache.page_size;
                if (g.t0 + t >= g.t1 || slot >= g.end) return a.cache.n_pages * a.Hkv;
                const int pg = a.cache.table[(int64_t)g.b * a.cache.max_pages + lp];
                if (pg >= 0 && pg < a.cache.n_pages) return pg * a.Hkv + g.h;
                atomicOr(a.status, ST_DEVICE);
                return a.cache.n_pages * a.Hkv;  // past the pool: the box reads as zeros
            };
            int z0 = place(0), z1 = z0, z2 = z0;  // of tiles t, t + 1, t + 2, as the loaders'
#pragma unroll 1
            for (int l = 0; l < 2 * nt; ++l) {
                const bool val = tile_is_value(l, nt);
                const int tt = tile_number(l, nt);
                if (!val) {
                    z0 = z1;
                    z1 = l == 0 ? z0 : z2;
                    z2 = place(tt + 1);
                }
                if (reuse && !(ok = wait(&st.empty[pos.slot], pos.phase ^ 1u))) break;
                if (!by_tma(a, g, tt, val)) {
                    pos.skip(1);
                    reuse |= pos.slot == 0;
                    continue;
                }
                // (rows past the item's end are zeros or whatever the cache holds: hidden from everyone, and
                // the loaders look through the values of tiles with nodes)
                const bool look = val && (g.t0 + tt + 1) * kTcTile > g.s.P;
                uint64_t* full = look ? &st.landed[pos.slot] : &st.full[pos.slot];
                if (lane == 0) {
                    mbar_arrive_expect_tx(full, TB);
                    if (!look) mbar_arrive_n(full, 127);  // in the place of the loaders' 128 arrivals
                }
                __syncwarp();
                const uint32_t phase = look ? landed >> pos.slot & 1u : pos.phase;
                sent = (sent & ~(0x10100u << pos.slot)) | 1u << pos.slot | phase << (8 + pos.slot) | (uint32_t)look << (16 + pos.slot);
                landed ^= (uint32_t)look << pos.slot;
                if (half < HD / 64) {
                    const int slot = (g.t0 + tt) * kTcTile + box * br;
                    const int y = a.cache.page_size ? slot % a.cache.page_size : slot;
                    tma_load_3d(smem_u32(ring) + pos.slot * TB + half * 16384 + box * br * 128, val ? &vmap : &kmap, half * 64, y,
                                !val || tt == nt - 1 ? z1 : z0, full);
                }
                pos.skip(1);
                reuse |= pos.slot == 0;
            }
        }
        while (a.box_rows <= 0 && next(g)) {}
    } else if (warp < 8) {  // ---- softmax
        const int gs = warp >> 2, wl = warp & 3;
        const uint32_t lanes = (uint32_t)(wl * 32) << 16;
        const uint32_t ts = tmem + gs * 128 + lanes, to = tmem + 256 + gs * 128 + lanes;
        const float scale2 = a.scale * kLog2e;
        uint32_t ns = 0, nj = 0;  // score blocks taken, joins of the streams
        // the warp's part of segment s's queries: rows of its own block, or half of the only one
        auto queries = [&](const Segment& s) {
            if (a.q_tma) return;  // (the planner's)
            if (s.weight == 2 || gs == 0)
                load_q<HD>(a, s, s.m * kAttnItemRows + gs * 128 + wl * 32, qbuf + gs * TB, wl, lane);
            if (a.q_vec) {
                cp_async_arrive(&st.qfull);
            } else {
                fence_async_proxy();
                mbar_arrive(&st.qfull);
            }
        };
        // e4m3: the warp's rows of segment number n's queries (as they have arrived) split for the product
        // (the MMA warps' proxy fence orders these writes before their reads)
        auto split = [&](const Segment& s, uint32_t n) -> bool {
            if constexpr (Q8) {
                if (!wait(&st.qfull, n)) return false;
                if (s.weight == 2 || gs == 0) {
                    query_scales[((n & 1) * 2 + gs) * 128 + wl * 32 + lane] = split_query_row<HD>(qbuf + gs * TB, wl * 32 + lane);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&st.qready);
            }
            return true;
        };
        uint32_t ktile = 0;  // the segment's first key tile (of kTcScales)
        Segment g2;  // the segment after this one, once its queries are on their way
        bool more = next(g2);
        if (more) {
            queries(g2);
            ok = split(g2, 0);
        }
        while (more && ok) {
            g = g2;
            const uint32_t cur = seg - 1;  // this segment's number
            const int nt = g.t1 - g.t0;
            const bool pair = g.weight == 2;
            const int row = g.m * kAttnItemRows + (pair ? gs * 128 : 0) + wl * 32 + lane;  // of the item's head
            const int node = row / a.G;
            const bool live = row < g.rows;
            const bool idle = row - lane >= g.rows;  // the whole warp
            const float* qscale = query_scales + ((cur & 1) * 2 + (pair ? gs : 0)) * 128 + wl * 32 + lane;
            float m = -INFINITY, sum = 0.f;  // reference maximum (log2 units), sum of 2^(s - m)
#pragma unroll 1
            for (int tt = pair ? 0 : gs; tt < nt; tt += pair ? 1 : 2) {
                const int tile = g.t0 + tt;
                const bool tail = (tile + 1) * kTcTile > g.s.P;  // some slots are nodes'
                ulonglong2 see = make_ulonglong2(0ull, 0ull);
                if (tail && live) see = seen_bits(a, g, node, tile * kTcTile);  // (while the scores are on their way)
                // (of a long causal run, most tiles are seen whole by all of the warp's rows)
                const bool hide = tail && __any_sync(0xffffffffu, live && (see.x & see.y) != ~0ull);
                if (!(ok = wait(&st.sfull[gs], ns))) break;
                ++ns;
                tc_fence_after();
                if (!idle) {
                    if (hide) {  // hidden scores become -inf
#pragma unroll 1
                        for (int c = 0; c < kTcTile; c += 32) {
                            const uint32_t bits = (uint32_t)((c < 64 ? see.x : see.y) >> (c & 32));
                            uint32_t x[32];
                            tc_ld32_start(ts + c, x);
                            tc_ld32_wait(x);
#pragma unroll
                            for (int e = 0; e < 32; ++e) x[e] = bits >> e & 1u ? x[e] : 0xFF800000u;
                            tc_st16(ts + c, x);
                            tc_st16(ts + c + 16, x + 16);
                        }
                        tc_wait_st();
                    }
                    softmax_row<HD, Q8>(ts, to, Q8 ? scale2 * *qscale : scale2,
                                        tt < 2 && (tt == 0 || !pair), key_scales + (ktile + tt) % kTcScales * kTcTile, m, sum);
                    tc_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&st.pfull[gs]);
            }
            // the next segment's queries may come once this one's scores are all done
            if (!ok) break;
            more = next(g2);
            if (more && !a.q_tma) {
                if (!(ok = wait(&st.qempty, cur))) break;
                queries(g2);
            }
            if (more && !(ok = split(g2, cur + 1))) break;
            ktile += nt;
            // ---- the segment's result
            if (!(ok = wait(&st.odone[gs], cur))) break;
            if (!pair && !(ok = wait(&st.odone[gs ^ 1], cur))) break;
            tc_fence_after();
            float f0 = 1.f, f1 = 0.f;  // weights of this stream's block, and of the other's (alternating)
            const bool join = !pair && nt > 1;
            if (join) {
                if (nj > 0 && !(ok = wait(&st.mlfree, nj - 1))) break;
                st.ml[gs][wl * 32 + lane] = make_float2(m, sum);
                __syncwarp();
                if (lane == 0) mbar_arrive(&st.mlfull);
                if (!(ok = wait(&st.mlfull, nj))) break;
                const float2 o = st.ml[gs ^ 1][wl * 32 + lane];
                __syncwarp();
                if (lane == 0) mbar_arrive(&st.mlfree);
                const float mn = fmaxf(m, o.x), ms = mn == -INFINITY ? 0.f : mn;
                f0 = exp2f(m - ms);
                f1 = exp2f(o.x - ms);
                sum = sum * f0 + o.y * f1;
                m = mn;
            }
            nj += join;
            // (a joined block's columns are shared out between the streams' warps)
            if (!idle && (pair || join || gs == 0)) {
                // A lane's row leaves 16 columns at a time, as whole sectors: of the output's row, or of the
                // partial's, where a warp's 32 rows of 4 columns are 512 bytes in a row.
                const int head = g.h * a.G + row % a.G;
                const int64_t pr = ((int64_t)blockIdx.x * 2 + g.slot) * kAttnItemRows + (row - g.m * kAttnItemRows);
                float* part = a.part_o + ((int64_t)blockIdx.x * 2 + g.slot) * (kAttnItemRows * HD) + (row - g.m * kAttnItemRows) * 4;
                bf16_t* dst = (bf16_t*)a.out.p + g.b * a.out.batch + (int64_t)node * a.out.token + (int64_t)head * a.out.head;
                // o = f0 u + f1 v with v the other stream's block.
                // Zero sums: a row that sees nothing, whose block may hold anything.
                const float norm = g.whole ? sum == 0.f ? 0.f : 1.f / sum : 1.f;
                f0 *= norm;
                f1 *= norm;
                const bool zero = g.whole && sum == 0.f;
#pragma unroll 1
                for (int c = join && gs ? HD / 2 : 0; c < (join && !gs ? HD / 2 : HD); c += 16) {
                    uint32_t u[16];
                    tc_ld16_start(to + c, u);
                    if (join) {
                        uint32_t v[16];
                        tc_ld16_start(tmem + 256 + (gs ^ 1) * 128 + lanes + c, v);
                        tc_ld16_wait(u);
                        tc_ld16_wait(v);
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            u[e] = __float_as_uint(fmaf(__uint_as_float(v[e]), f1, __uint_as_float(u[e]) * f0));
                    } else {
                        tc_ld16_wait(u);
#pragma unroll
                        for (int e = 0; e < 16; ++e) u[e] = __float_as_uint(__uint_as_float(u[e]) * f0);
                    }
                    if (!live) continue;
                    if (!g.whole) {
#pragma unroll
                        for (int e = 0; e < 16; e += 4)
                            *reinterpret_cast<uint4*>(part + (c + e) * kAttnItemRows) = make_uint4(u[e], u[e + 1], u[e + 2], u[e + 3]);
                        continue;
                    }
                    uint32_t w[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        w[e] = zero ? 0u : pack_bf16(__uint_as_float(u[2 * e]), __uint_as_float(u[2 * e + 1]));
                    if (a.out_vec == 2) {
                        st_global_32(dst + c, w);
                    } else if (a.out_vec) {
                        *reinterpret_cast<uint4*>(dst + c) = make_uint4(w[0], w[1], w[2], w[3]);
                        *reinterpret_cast<uint4*>(dst + c + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; ++e) dst[c + e].bits = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
                    }
                }
                if (live && (pair || gs == 0)) {
                    if (!g.whole)
                        *reinterpret_cast<float2*>(a.part_ml + 2 * pr) = make_float2(m, sum);
                    else if (a.lse)
                        a.lse[((int64_t)g.b * a.T + node) * a.H + head] =
                            sum == 0.f ? -INFINITY : m * 0.6931471805599453f + logf(sum);
                }
                if (live && !zero && *(volatile int*)&st.odd[cur & 7])
                    put_odd_columns<HD, Q8>(a, g, node, head, g.whole ? (void*)dst : (void*)part, join && gs ? HD / 2 : 0, join && !gs ? HD / 2 : HD);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                // (the next segment's first value tile is not released yet, so the ring lets the loaders
                // be at most three segments ahead; the other stream is at most one behind)
                if (warp == 0) st.odd[(cur + 4) & 7] = 0;
                mbar_arrive(&st.ofree);
            }
        }
        cp_async_wait_all();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 12) tc_dealloc(tmem, 512);
    // Leave with no copy in flight. (Otherwise every copy has been waited for and used.)
    if (*(volatile int*)&st.abort && sent) {
        constexpr int64_t kLimit = 100000000;  // ns
        if (warp == 14) {
            mbar_wait(&st.qfull, (sent - 1) & 1u, a.status, kLimit);
        } else if (Q8) {
            for (uint32_t j = sent > (uint32_t)KS ? sent - KS : 0; j < sent; ++j)
                mbar_wait(&st.kfull[j % KS], (j / KS) & 1u, a.status, kLimit);
        } else {
            for (int k = 0; k < S; ++k)
                if (sent >> k & 1u) mbar_wait(sent >> (16 + k) & 1u ? &st.landed[k] : &st.full[k], sent >> (8 + k) & 1u, a.status, kLimit);
        }
    }
}

}  // namespace fe
