// How a matrix product is divided, by its sizes (host): the tiles of fe_gemm_tc.cu, the blocks of fe_gemm_few.cu
// and the tiles of fe_gemm_simt.cu.
#pragma once

#include <cstdint>

namespace fe {

// ---- tiles of 256 rows by pairs of CTAs --------------------------------------------------------
constexpr int kFinishWarps = 8;
constexpr int kTileM = 256, kSliceK = 64;
constexpr int kSliceA = 128 * kSliceK * 2;
constexpr int kTcRing = 192 * 1024, kTcStages = 8;
constexpr int kPairs = kFinishWarps * 8192;  // of the ring, for a gated gradient's products on their way

// the tile's width and what follows from it
struct TcWidth {
    int bn, b_bytes, stages;  // B's bytes of a slice in a CTA, slices in flight
};

// results: gated, a pair of products a tile; twice, two results of one B; grad, a gated gradient; b_t: B by its summed index
inline int64_t tc_tiles(int64_t M, int N, bool gated, bool twice, int bn) {
    const int width = gated ? bn / 2 : bn;
    return (M + kTileM - 1) / kTileM * (twice ? 2 : 1) * ((N + width - 1) / width);
}
// The width: rounds of tiles, each of its columns' time, or of its copies' where that is more (a column's products
// of a slice take as long as the copy of 134 bytes), and of some 16 columns' for its start. B by its summed
// index comes in whole groups of 64 columns: there a width of 160 (5120 x 5120 from 4093 rows, 9 rounds)
// took 174 us and 256 (6 rounds) 128 us.
inline TcWidth tc_width(int64_t M, int N, bool gated, bool twice, bool grad, bool b_t, int num_sms) {
    const int64_t pairs = num_sms / 2;
    TcWidth shape{};
    int64_t best = 0;
    for (int w = 256; w >= 128; w -= 32) {
        const int b_bytes = b_t ? (w / 2 + 63) / 64 * 8192 : w / 2 * 128, copies = (kSliceA + b_bytes) / 134;
        const int64_t cost = (tc_tiles(M, N, gated, twice, w) + pairs - 1) / pairs * ((w > copies ? w : copies) + 16);
        if (!best || cost < best) {
            best = cost;
            shape.bn = w;
            shape.b_bytes = b_bytes;
        }
    }
    shape.stages = (kTcRing - (grad ? kPairs : 0)) / (kSliceA + shape.b_bytes);
    if (shape.stages > kTcStages) shape.stages = kTcStages;
    return shape;
}

// ---- blocks of 128 weight rows by clusters -----------------------------------------------------
constexpr int kFewRows = 128, kFewStages = 12, kFewMost = 8;
constexpr int kPartRow = kFewRows + 4;     // floats of a token's sums in shared memory
constexpr int kFewSmem = 224 * 1024;       // of an SM, for its CTAs' rings

struct FewArgs {
    int nt, stages, stage_bytes, ranks;
};

inline FewArgs few_plan(int64_t M, int N, int K, bool gated, int num_sms, int* smem) {
    const int rows = gated ? 64 : 128, slices = (K + 63) / 64;
    const int64_t blocks = ((int64_t)N + rows - 1) / rows;
    FewArgs f{};
    f.nt = (int)(M + 15) / 16 * 16;
    // How many CTAs share a block: the busiest SM's CTAs, each with its slices and some four slices' time
    // for its start and the join
    int64_t best = 0;
    for (int r = 1; r <= kFewMost && r <= slices; r *= 2) {
        const int64_t per = (blocks * r + num_sms - 1) / num_sms, cost = per * ((slices + r - 1) / r + 4);
        if (!best || cost < best) {
            best = cost;
            f.ranks = r;
        }
    }
    f.stage_bytes = 16384 + (f.nt * 128 + 1023) / 1024 * 1024;
    // the rings of the CTAs that an SM holds at once, up to four, share its memory
    const int64_t per = (blocks * f.ranks + num_sms - 1) / num_sms;
    const int held = per < 4 ? (int)per : 4, mine = (slices + f.ranks - 1) / f.ranks;
    const int part = (int)M * kPartRow * 4;
    f.stages = (kFewSmem / held - 4096) / f.stage_bytes;
    if (f.stages > kFewStages) f.stages = kFewStages;
    if (f.stages > mine) f.stages = mine;
    if (f.stages < 2) f.stages = 2;
    *smem = f.stages * f.stage_bytes;
    *smem = (*smem > part ? *smem : part) + 1024;
    return f;
}

// ---- tiles on the CUDA cores -------------------------------------------------------------------
// too few large tiles (128 x 128) to occupy the GPU: a quarter of the size
inline bool simt_large(int64_t M, int N, bool gated, bool twice, int num_sms) {
    const int64_t big = ((M + 127) / 128) * ((N + (gated ? 63 : 127)) / (gated ? 64 : 128)) * (twice ? 2 : 1);
    return big >= num_sms && M > 64;
}

}  // namespace fe
