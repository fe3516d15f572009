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
    // Set by Place::find: short items (of JOIN tiles at most, on average), no more of them than CTAs,
    // are not split; every item then counts as one unit, and CTA c has item c.
    bool whole = false;
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

// ROWS rows an item, TN slots a tile; PAIR: an item of more than 128 rows costs two units a tile.
// An item begins with OVER units that hold no tile: what starting and finishing it costs a CTA, in
// units, so that a CTA with many short items does not end after one with few long ones. JOIN: about
// how many tiles joining a split costs: items of that many on average, no more of them than CTAs, are
// not split. Above it splitting pays (one token over 199 float32 slots, 8 items of 4 tiles of 64: 20 us
// split, 36 whole). TAIL: what a tile that reaches into the nodes' slots costs an item of two units a
// tile besides (masks, values to look through).
// Units are counted in 32 bits (the launch refuses shapes that could pass 2^31): this runs once a
// CTA before anything else can start, and short code is what it takes to be quick.
template <int ROWS, int TN, bool PAIR, int OVER, int JOIN, int TAIL>
struct Plan {
    static constexpr int kOver = OVER, kJoin = JOIN;
    __host__ __device__ __forceinline__ static int blocks(int rows) { return (rows + ROWS - 1) / ROWS; }
    __device__ __forceinline__ static int weight(int rows, int m) { return PAIR && rows - m * ROWS > 128 ? 2 : 1; }
    // slots that block m's rows may see: [0, end)
    __device__ __forceinline__ static int end(const PlanArgs& a, SeqLen s, int m) {
        if (!a.causal) return s.P + s.n;
        const int last = min((m + 1) * ROWS, s.n * a.G) - 1;
        return s.P + last / a.G + 1;
    }
    __device__ __forceinline__ static int tiles(const PlanArgs& a, SeqLen s, int m) {
        return (int)((uint32_t)(end(a, s, m) + TN - 1) / TN);
    }
    // units of one KV head of a sequence
    __device__ __forceinline__ static int head_units(const PlanArgs& a, SeqLen s) {
        const int rows = s.n * a.G, nb = blocks(rows);
        if (a.whole || nb == 0) return nb;
        if (!a.causal) {  // every block but the last is full
            const int full = weight(ROWS, 0), last = weight(rows, nb - 1), nt = tiles(a, s, 0);
            return nb * OVER + nt * ((nb - 1) * full + last) + tail(s, nt) * ((nb - 1) * (full - 1) + last - 1);
        }
        int u = nb * OVER;
#pragma unroll 1
        for (int m = 0; m < nb; ++m) {
            const int w = weight(rows, m), nt = tiles(a, s, m);
            u += nt * w + tail(s, nt) * (w - 1);
        }
        return u;
    }
    // what the first t tiles' share in the nodes' slots costs besides, for an item of weight 2
    __device__ __forceinline__ static int tail(SeqLen s, int t) { return TAIL ? TAIL * max(t - s.P / TN, 0) : 0; }
    // units of an item of nt tiles of weight w = 1 or 2; the unit where tile t starts
    __device__ __forceinline__ static int units(const PlanArgs& a, SeqLen s, int w, int nt) {
        return a.whole ? 1 : OVER + w * nt + tail(s, nt) * (w - 1);
    }
    __device__ __forceinline__ static int tile_unit(const PlanArgs& a, SeqLen s, int s0, int w, int t) {
        return a.whole ? s0 : s0 + OVER + w * t + tail(s, t) * (w - 1);
    }
    // first tile of an item with first unit s0 that starts at unit u0 or later
    __device__ __forceinline__ static int first_tile(const PlanArgs& a, SeqLen s, int s0, int w, int nt, int u0) {
        if (a.whole) return u0 <= s0 ? 0 : nt;
        const int d = u0 - s0 - OVER, tp = s.P / TN;
        if (d <= 0) return 0;
        int t = (d + w - 1) >> (w - 1);
        if (TAIL && w == 2 && t > tp) t = tp + (d - 2 * tp + 1 + TAIL) / (2 + TAIL);
        return min(t, nt);
    }
    // whether every call of T nodes with G heads to a KV head keeps its units within 32 bits
    static bool fits(int B, int Hkv, int T, int G, int max_seq) {
        const double items = (double)B * Hkv * (double)(((int64_t)T * G + ROWS - 1) / ROWS);
        return items * (2.0 * (max_seq / TN + 1 + OVER) + TAIL * (T / TN + 2.0)) < 2147483647.0;
    }
};

// The line of U units cut into G CTAs: CTA c has the units [begin(c), begin(c + 1)), begin(c) =
// floor(c U / G).
struct Cut {
    int q, r, G;
    __device__ __forceinline__ Cut(int U, int ncta) : q(U / ncta), r(U - U / ncta * ncta), G(ncta) {}
    __device__ __forceinline__ int begin(int c) const { return c * q + (int)((uint32_t)(c * r) / (uint32_t)G); }
    // the last CTA whose begin is <= s: a guess in float32 (off by one at most), corrected
    __device__ __forceinline__ int owner(int s) const {
        int c = min((int)((float)s * (float)G / ((float)q * (float)G + (float)r)), G - 1);
        while (c > 0 && begin(c) > s) --c;
        while (c + 1 < G && begin(c + 1) <= s) ++c;
        return c;
    }
};

// A CTA's share of an item: tiles [t0, t1).
struct Segment {
    int b, h, m, rows, weight;
    SeqLen s;
    int end, t0, t1;
    int whole;  // the item has no other share
    int slot;   // where its partial goes: 0 when an earlier CTA began the item, else 1
};

// Where CTA c's units begin: the cut of the line and the item that holds unit cut.begin(c).
// Found by a whole warp together, every lane with the same result.
template <typename PL>
struct Place {
    Cut cut;
    bool found;  // false: no unit at or past the beginning
    int b, h, m, s0;  // the item and its first unit
    SeqLen s;

    __device__ __forceinline__ static Place find(PlanArgs& a, int c, int ncta, bool* bad = nullptr) {
        const int lane = threadIdx.x & 31;
        SeqLen sl;
        int hu = 0, U = 0, items = 0;
#pragma unroll 1
        for (int b0 = (a.B - 1) & ~31; b0 >= 0; b0 -= 32) {  // (ends with the first 32's in sl and hu)
            sl = b0 + lane < a.B ? seq_len(a, b0 + lane, bad) : SeqLen{0, 0};
            hu = PL::head_units(a, sl);
            U += hu;
            items += PL::blocks(sl.n * a.G);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            U += __shfl_xor_sync(0xffffffffu, U, o);
            items += __shfl_xor_sync(0xffffffffu, items, o);
        }
        U *= a.Hkv;
        items *= a.Hkv;
        a.whole = items <= ncta && U <= items * (PL::kOver + PL::kJoin);
        if (a.whole) {
            U = items;
            hu = PL::blocks(sl.n * a.G);
        }
        Place p{Cut(U, a.whole ? max(items, 1) : ncta), false, 0, 0, 0, 0, SeqLen{0, 0}};
        if (c >= p.cut.G) return p;
        const int u0 = p.cut.begin(c);
        if (u0 >= U) return p;
        // the sequence that holds unit u0: the first whose units end past it
        int base = 0;
#pragma unroll 1
        for (int b0 = 0; b0 < a.B; b0 += 32) {
            if (b0) {
                sl = b0 + lane < a.B ? seq_len(a, b0 + lane) : SeqLen{0, 0};
                hu = PL::head_units(a, sl);
            }
            int inc = hu * a.Hkv;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += v;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, base + inc > u0);
            if (hit) {
                const int l = __ffs(hit) - 1;
                p.found = true;
                p.b = b0 + l;
                p.s.P = __shfl_sync(0xffffffffu, sl.P, l);
                p.s.n = __shfl_sync(0xffffffffu, sl.n, l);
                const int head = __shfl_sync(0xffffffffu, hu, l);
                p.s0 = base + __shfl_sync(0xffffffffu, inc, l) - head * a.Hkv;
                p.h = (u0 - p.s0) / head;
                p.s0 += p.h * head;
                break;
            }
            base += __shfl_sync(0xffffffffu, inc, 31);
        }
        // the block of the head
#pragma unroll 1
        while (true) {
            const int w = PL::units(a, p.s, PL::weight(p.s.n * a.G, p.m), PL::tiles(a, p.s, p.m));
            if (p.s0 + w > u0) return p;
            p.s0 += w;
            ++p.m;
        }
    }
};

// Walks a CTA's segments; used by a whole warp, every lane holding the same state.
template <typename PL>
struct SegmentWalk {
    Cut cut;
    int u0, u1, pos;  // the CTA's units; first unit of the current item
    int b, h, m;
    SeqLen s;

    __device__ __forceinline__ SegmentWalk() : cut(0, 1) {}
    __device__ __forceinline__ void init(PlanArgs& a, int cta, int ncta, bool* bad = nullptr) {
        const Place<PL> p = Place<PL>::find(a, cta, ncta, bad);
        cut = p.cut;
        u0 = p.cut.begin(cta);
        u1 = p.cut.begin(cta + 1);
        b = p.found ? p.b : a.B;
        h = p.h;
        m = p.m;
        pos = p.s0;
        s = p.s;
    }
    // What the join has to know of this CTA; after the last next(), with the last segment and whether
    // some segment's slot was 0.
    __device__ __forceinline__ SplitDesc desc(const PlanArgs& a, bool any, const Segment& g, bool continues) const {
        SplitDesc d{};
        d.has0 = continues;
        d.last = -1;
        if (any && !g.whole && g.slot == 1) {  // an item begins here and goes on
            const int nt = PL::tiles(a, g.s, g.m), w = g.weight, p = pos - PL::units(a, g.s, w, nt);  // (pos: past the item)
            d.b = g.b;
            d.h = g.h;
            d.m = g.m;
            d.rows = g.rows;
            d.last = cut.owner(PL::tile_unit(a, g.s, p, w, nt - 1));
        }
        return d;
    }
    // The next segment with at least one tile; false at the end.
    __device__ __forceinline__ bool next(const PlanArgs& a, Segment& g) {
#pragma unroll 1
        while (b < a.B && pos < u1) {
            const int rows = s.n * a.G;
            bool got = false;
            if (rows > 0) {
                const int w = PL::weight(rows, m), nt = PL::tiles(a, s, m);
                g.t0 = PL::first_tile(a, s, pos, w, nt, u0);
                g.t1 = PL::first_tile(a, s, pos, w, nt, u1);
                got = g.t0 < g.t1;
                if (got) {
                    g.b = b;
                    g.h = h;
                    g.m = m;
                    g.rows = rows;
                    g.weight = w;
                    g.s = s;
                    g.end = PL::end(a, s, m);
                    g.whole = g.t0 == 0 && g.t1 == nt;
                    g.slot = g.t0 == 0 ? 1 : 0;
                }
                pos += PL::units(a, s, w, nt);
            }
            if (++m >= PL::blocks(rows)) {
                m = 0;
                if (++h >= a.Hkv) {
                    h = 0;
                    if (++b < a.B) s = seq_len(a, b);
                }
            }
            if (got) return true;
        }
        return false;
    }
};

// ---- the kernels' schedules ------------------------------------------------------------------
constexpr int kTcTile = 128, kSimtTile = 64;

// What an item's start and finish cost, in tiles of 128 rows: 4, and 6 where the queries are split too
// (e4m3, 32 x 49 nodes: 111 us with 4, 104 with 6, 105 with 8; bfloat16, 2 x 1021 causal tokens: 112
// us with 4 or 5; 3 x 700: 69 us with 4, 71 with 5). And what a tile with nodes costs two streams
// besides: half a tile's time over bfloat16 (3 x 700 causal tokens: 74 us without, 69 with; 4096 from
// an empty cache: 169 without, 173 with), nothing over e4m3, whose values all pass the loaders (139
// us without, 141 with, 2 x 1021 tokens).
template <bool Q8>
using TcPlan = Plan<kAttnItemRows, kTcTile, true, Q8 ? 6 : 4, 6, Q8 ? 0 : 1>;
// The float32 kernel's, of 16 NI rows an item.
template <int NI>
using SimtPlan = Plan<16 * NI, kSimtTile, false, 1, 2, 0>;

// Whether the schedule that a call runs on can count the work of every call of its shape.
inline bool attn_plan_fits(fe_dtype dtype, fe_dtype cache_dtype, int B, int Hkv, int T, int G, int max_seq) {
    if (dtype == FE_F32) return SimtPlan<4>::fits(B, Hkv, T, G, max_seq);  // (the variants of fewer rows hold all of an item's)
    return cache_dtype == FE_E4M3 ? TcPlan<true>::fits(B, Hkv, T, G, max_seq) : TcPlan<false>::fits(B, Hkv, T, G, max_seq);
}

}  // namespace fe
