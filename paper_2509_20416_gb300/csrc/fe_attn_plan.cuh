// How the attention's work is divided: one schedule, computed on the device from the lengths,
// that the attention kernels and the kernel joining their partial results share.
//
// An item is (sequence b, KV head h, block m of up to ROWS query rows of that head); row r of a
// (b, h) is node r / G, query head h G + r % G. An item runs over tiles of TN slots from 0 to
// the last slot that any of its rows may see. Items in the order (b, h, m) form one line of
// units, a tile of an item costing `weight` units, and CTA c of G takes the tiles that start in
// units [c U / G, (c + 1) U / G): every CTA gets the same work whatever the lengths, a long
// sequence is split over many CTAs and short ones share one. An item whose tiles all fall to one
// CTA is finished there; otherwise each CTA leaves a partial result that the join sums in CTA
// order, so the result does not depend on timing.
#pragma once

#include "fe_target_common.cuh"

namespace fe {

struct PlanArgs {
    int B, T, Hkv, G, max_seq;
    const int *prefix, *nodes;
    bool causal;
};

__device__ __forceinline__ PlanArgs plan_args(const TreeAttnArgs& a) {
    return PlanArgs{a.B, a.T, a.Hkv, a.G, a.cache.max_seq, a.prefix, a.nodes, a.mask == nullptr};
}

// Prefix and node count of sequence b; a sequence out of range has no nodes (and *bad is set).
struct SeqLen {
    int P, n;
};
__device__ __forceinline__ SeqLen seq_len(const PlanArgs& a, int b, bool* bad = nullptr) {
    SeqLen s;
    s.P = a.prefix[b];
    s.n = a.nodes ? a.nodes[b] : a.T;
    if (s.P < 0 || s.n < 0 || s.n > a.T || (int64_t)s.P + s.n > a.max_seq) {
        if (bad) *bad = true;
        s.P = s.n = 0;
    }
    return s;
}

// ROWS rows an item, TN slots a tile; PAIR: an item of more than 128 rows costs two units a tile
template <int ROWS, int TN, bool PAIR>
struct Plan {
    __device__ __forceinline__ static int blocks(int rows) { return (rows + ROWS - 1) / ROWS; }
    __device__ __forceinline__ static int weight(int rows, int m) { return PAIR && rows - m * ROWS > 128 ? 2 : 1; }
    // slots that block m's rows may see: [0, end)
    __device__ __forceinline__ static int end(const PlanArgs& a, SeqLen s, int m) {
        if (!a.causal) return s.P + s.n;
        const int last = min((m + 1) * ROWS, s.n * a.G) - 1;
        return s.P + last / a.G + 1;
    }
    __device__ __forceinline__ static int tiles(const PlanArgs& a, SeqLen s, int m) {
        return (end(a, s, m) + TN - 1) / TN;
    }
    // units of one KV head of a sequence
    __device__ __forceinline__ static int64_t head_units(const PlanArgs& a, SeqLen s) {
        const int rows = s.n * a.G, nb = blocks(rows);
        if (nb == 0) return 0;
        if (!a.causal) {  // every block but the last is full
            return (int64_t)tiles(a, s, 0) * ((int64_t)(nb - 1) * weight(ROWS, 0) + weight(rows, nb - 1));
        }
        int64_t u = 0;
        for (int m = 0; m < nb; ++m) u += (int64_t)tiles(a, s, m) * weight(rows, m);
        return u;
    }
    // CTA c's first unit
    __device__ __forceinline__ static int64_t begin(int64_t c, int64_t U, int G) { return c * U / G; }
    // the CTA that owns the tile starting at unit s
    __device__ __forceinline__ static int owner(int64_t s, int64_t U, int G) { return (int)(((s + 1) * G - 1) / U); }
    // tiles of an item (first unit s0, weight w, nt tiles) that start in units [u0, u1)
    __device__ __forceinline__ static int first_tile(int64_t s0, int w, int nt, int64_t u0) {
        if (u0 <= s0) return 0;
        const int64_t t = (u0 - s0 + w - 1) / w;
        return t < nt ? (int)t : nt;
    }
};

// Sum of head_units * Hkv over all sequences; called by a whole warp.
template <typename PL>
__device__ __forceinline__ int64_t plan_total(const PlanArgs& a, bool* bad = nullptr) {
    int64_t u = 0;
    for (int b = threadIdx.x & 31; b < a.B; b += 32) u += PL::head_units(a, seq_len(a, b, bad));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) u += __shfl_xor_sync(0xffffffffu, u, o);
    return u * a.Hkv;
}

// A CTA's share of an item: tiles [t0, t1) of nt.
struct Segment {
    int b, h, m, rows, weight;
    SeqLen s;
    int end, t0, t1, nt;
    bool whole;  // the item has no other share
    int slot;    // where its partial goes: 0 when an earlier CTA began the item, else 1
};

// Walks a CTA's segments. Every lane of a warp holds the same state (init is collective).
template <typename PL>
struct SegmentWalk {
    int64_t u0, u1, pos;  // the CTA's units; first unit of the current item
    int b, h, m;
    SeqLen s;
    bool done;

    __device__ __forceinline__ void init(const PlanArgs& a, int cta, int ncta, bool* bad = nullptr) {
        const int lane = threadIdx.x & 31;
        const int64_t U = plan_total<PL>(a, bad);
        u0 = PL::begin(cta, U, ncta);
        u1 = PL::begin(cta + 1, U, ncta);
        done = u0 >= u1;
        b = h = m = 0;
        pos = 0;
        s = SeqLen{0, 0};
        if (done) return;
        // the sequence that holds unit u0: the last whose first unit is <= u0 (and has units)
        int64_t base = 0;
        for (int b0 = 0; b0 < a.B; b0 += 32) {
            const int bb = b0 + lane;
            const SeqLen sl = bb < a.B ? seq_len(a, bb) : SeqLen{0, 0};
            const int64_t hu = PL::head_units(a, sl), w = hu * a.Hkv;
            int64_t inc = w;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t v = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += v;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, base + inc > u0);
            if (hit) {
                const int l = __ffs(hit) - 1;
                b = b0 + l;
                s.P = __shfl_sync(0xffffffffu, sl.P, l);
                s.n = __shfl_sync(0xffffffffu, sl.n, l);
                const int64_t head = __shfl_sync(0xffffffffu, hu, l);
                pos = base + __shfl_sync(0xffffffffu, inc - w, l);
                h = (int)((u0 - pos) / head);
                pos += h * head;
                break;
            }
            base += __shfl_sync(0xffffffffu, inc, 31);
        }
        m = 0;
        while (true) {  // the block that holds u0
            const int64_t w = units(a);
            if (pos + w > u0) break;
            pos += w;
            ++m;
        }
    }
    __device__ __forceinline__ int64_t units(const PlanArgs& a) const {
        return (int64_t)PL::tiles(a, s, m) * PL::weight(s.n * a.G, m);
    }
    // The next segment with at least one tile; false at the end.
    __device__ __forceinline__ bool next(const PlanArgs& a, Segment& g) {
        while (!done) {
            const int rows = s.n * a.G;
            bool got = false;
            if (PL::blocks(rows) > 0) {
                const int w = PL::weight(rows, m), nt = PL::tiles(a, s, m);
                g.t0 = PL::first_tile(pos, w, nt, u0);
                g.t1 = PL::first_tile(pos, w, nt, u1);
                got = g.t0 < g.t1;
                if (got) {
                    g.b = b;
                    g.h = h;
                    g.m = m;
                    g.rows = rows;
                    g.weight = w;
                    g.s = s;
                    g.nt = nt;
                    g.end = PL::end(a, s, m);
                    g.whole = g.t0 == 0 && g.t1 == nt;
                    g.slot = g.t0 == 0 ? 1 : 0;
                }
                pos += (int64_t)nt * w;
            }
            if (++m >= PL::blocks(rows)) {
                m = 0;
                if (++h >= a.Hkv) {
                    h = 0;
                    if (++b < a.B) s = seq_len(a, b);
                }
            }
            if (b >= a.B || pos >= u1) done = true;
            if (got) return true;
        }
        return false;
    }
};

}  // namespace fe
