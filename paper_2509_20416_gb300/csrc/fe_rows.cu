// Row operators of the target side: rotary positions (fe_rope), the cache's write with its
// rotation and quantisation (fe_cache_write), its read (fe_cache_read) and the move of
// accepted rows (fe_cache_keep). All are bound by memory traffic: each row is read once and
// written once, in 16-byte accesses where the caller's alignment allows, and everything
// between (rotation, row maximum, rounding) happens in registers.
//
// A row of hd elements is held by a group of hd / (2 V) consecutive lanes, V the elements of 16
// bytes of the rows' type; each lane holds two vectors of V elements chosen so that a rotation's
// pairs meet in one lane: with rope_dim a multiple of 2 V, lane u of a HALF row holds vectors u
// and u + rope_dim / 2 V of the rotated part, and every other vector pair is (2 u, 2 u + 1).
// Other rope dimensions, and rows off 16-byte boundaries, take the element-wise variant (FAST
// = false), where a lane reads each element's partner itself.
#include "fe_target_common.cuh"

namespace fe {

namespace {

constexpr int kRowThreads = 256;

// cos and sin of pos * f_i in double precision (the argument reaches max_seq radians, where a
// float32 product would lose log2(max_seq) bits), times the amplitude, rounded once
__global__ void rope_table_kernel(float2* table, int max_seq, int pairs, const double* inv_freq, double amplitude) {
    const int64_t n = (int64_t)max_seq * pairs;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
        const double ang = (double)(i / pairs) * inv_freq[i % pairs];
        double s, c;
        sincos(ang, &s, &c);
        table[i] = make_float2((float)(c * amplitude), (float)(s * amplitude));
    }
}

// One lane's share of a row: element offsets of its two vectors, and its unit number.
template <int V>
struct Share {
    int e0, e1;
    __device__ __forceinline__ Share(int u, const RopeView& r) {
        const int ru = r.dim / (2 * V);  // units inside the rotated part
        const bool split = !r.interleaved && u < ru;
        e0 = V * (split ? u : 2 * u);
        e1 = V * (split ? u + ru : 2 * u + 1);
    }
};

// A lane's V pairs, (x[e], x[V + e]) or neighbours, by the angles whose (cos, sin) are t.
template <int V, bool NEIGHBOURS>
__device__ __forceinline__ void rotate_pairs(float* x, const float2* t) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
        float& a = x[NEIGHBOURS ? 2 * e : e];
        float& b = x[NEIGHBOURS ? 2 * e + 1 : V + e];
        const float ya = a * t[e].x - b * t[e].y, yb = b * t[e].x + a * t[e].y;
        a = ya;
        b = yb;
    }
}

// The same element by element, each partner read from the row itself.
template <typename ST>
__device__ __forceinline__ void rotate_elements(const ST* row, int e0, int e1, const RopeView& r, const float2* cs, float dir,
                                                float* x) {
    constexpr int V = Vec16<ST>::kN;
    const int half = r.dim / 2;
#pragma unroll
    for (int j = 0; j < 2 * V; ++j) {
        const int e = j < V ? e0 + j : e1 + j - V;
        if (e >= r.dim) continue;
        const bool first = r.interleaved ? !(e & 1) : e < half;
        const int pe = r.interleaved ? e ^ 1 : first ? e + half : e - half;
        const float2 t = __ldg(cs + (r.interleaved ? e >> 1 : first ? e : e - half));
        const float p = Storage<ST>::load(row, pe), s = t.y * dir;
        x[j] = first ? x[j] * t.x - p * s : x[j] * t.x + p * s;
    }
}

template <typename ST, bool FAST>
__device__ __forceinline__ void store_share(ST* row, int e0, int e1, const float* x) {
    constexpr int V = Vec16<ST>::kN;
    if (FAST) {
        *reinterpret_cast<uint4*>(row + e0) = pack16<ST>(x);
        *reinterpret_cast<uint4*>(row + e1) = pack16<ST>(x + V);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            store_one(row + e0 + j, x[j]);
            store_one(row + e1 + j, x[V + j]);
        }
    }
}

// The scale exponent c of a row whose largest finite magnitude is m: the smallest c >= -120
// with m <= 448 * 2^c (448 = 1.75 * 2^8), from m's bits.
__device__ __forceinline__ int scale_exp(float m) {
    const uint32_t u = __float_as_uint(m);
    return max((int)(u >> 23) - 135 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0), -120);
}
__device__ __forceinline__ float pow2(int c) { return __uint_as_float((uint32_t)(c + 127) << 23); }

// A group's row, 2 V elements a lane, to e4m3 at `out` and its scale.
template <int HD, int V>
__device__ __forceinline__ void quantise_share(const float* x, unsigned lanes, int e0, int e1, uint8_t* out, float* scale,
                                               bool first_lane) {
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < 2 * V; ++e) m = fmaxf(m, finite_f32(x[e]) ? fabsf(x[e]) : 0.f);
#pragma unroll
    for (int o = HD / (2 * V) / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(lanes, m, o));
    const int c = scale_exp(m);
    const float inv = pow2(-c);
    uint32_t w[V / 2];
#pragma unroll
    for (int e = 0; e < 2 * V; e += 4) {
        float y[4];
#pragma unroll
        for (int z = 0; z < 4; ++z)  // (a non-finite element becomes NaN)
            y[z] = finite_f32(x[e + z]) ? x[e + z] * inv : __uint_as_float(0x7FC00000u);
        w[e / 4] = f32x2_to_e4m3(y[0], y[1]) | (f32x2_to_e4m3(y[2], y[3]) << 16);
    }
    if (V == 8) {
        *reinterpret_cast<uint2*>(out + e0) = make_uint2(w[0], w[1]);
        *reinterpret_cast<uint2*>(out + e1) = make_uint2(w[V / 4], w[V / 4 + 1]);
    } else {
        *reinterpret_cast<uint32_t*>(out + e0) = w[0];
        *reinterpret_cast<uint32_t*>(out + e1) = w[V / 4];
    }
    if (first_lane) *scale = pow2(c);
}

// One group per job: four of a token's rotated heads, or two KV heads' key and value rows. Four rows
// a lane keep 128 bytes in flight (about what the memory's latency takes at two blocks an SM) and
// share the token's table row and address arithmetic. (Two rows a lane with 64-bit index divisions
// moved 2.5 TB/s at 32 thousand tokens of 64 + 8 heads; this 5.8 TB/s with rotation, quantisation and
// pages of 64, 216 us. The gradient of 16 thousand tokens' 40 float32 heads takes 97 us, 6.9 TB/s.)
template <typename ST, int HD, int CACHE, bool FAST>
__global__ void __launch_bounds__(kRowThreads, 3) rows_kernel(const __grid_constant__ RowsArgs a) {
    constexpr int V = Vec16<ST>::kN, GL = HD / (2 * V);
    const uint32_t ja = (a.HA + 3) / 4, jb = CACHE ? (a.HB + 1) / 2 : (a.HB + 3) / 4, J = ja + jb;
    const uint32_t group = blockIdx.x * (kRowThreads / GL) + threadIdx.x / GL;
    const int u = threadIdx.x % GL;
    if (group >= (uint32_t)(a.B * a.T) * J) return;  // (whole groups: the shuffles below stay inside one)
    const uint32_t token = group / J;
    const int j = (int)(group - token * J), b = (int)(token / (uint32_t)a.T), i = (int)(token - (uint32_t)b * a.T);
    const Share<V> sh(u, a.rope);
    // the group's lanes of the warp: they take every branch below together
    const unsigned lanes = ((1u << GL) - 1u) << ((threadIdx.x & 31) / GL * GL);

    const bool kv = CACHE && j >= (int)ja;
    int pos = 0;
    if (a.pos) pos = a.pos[token];
    if (kv) {  // (a row past n_rows[b] is none: its position may be anything)
        const int n = a.n_rows ? a.n_rows[b] : a.T;
        if (n < 0 || n > a.T) {
            if (u == 0) atomicOr(a.status, ST_DEVICE);
            return;
        }
        if (i >= n) return;
    }
    if (a.pos) {
        if (pos < 0 || pos >= a.rope.max_pos) {
            if (u == 0) atomicOr(a.status, ST_CAPACITY);
            return;
        }
    }
    const ST* src[4];
    int64_t crow = 0;
    int h0, heads;  // the job's first head, of how many
    const fe_rows& out = !CACHE && j >= (int)ja ? a.b_out : a.a_out;
    if (kv) {
        h0 = 2 * (j - (int)ja);
        heads = a.HB;
        if (!cache_row(a.cache, b, (int64_t)a.start[b] + i, crow, a.status)) return;
        const ST* k = (const ST*)a.b_in.p + b * a.b_in.batch + i * a.b_in.token + h0 * a.b_in.head;
        const ST* v = (const ST*)a.v_in.p + b * a.v_in.batch + i * a.v_in.token + h0 * a.v_in.head;
        const bool two = h0 + 1 < heads;
        src[0] = k;
        src[1] = v;
        src[2] = two ? k + a.b_in.head : nullptr;
        src[3] = two ? v + a.v_in.head : nullptr;
    } else {
        const bool second = !CACHE && j >= (int)ja;
        const fe_rows& in = second ? a.b_in : a.a_in;
        h0 = 4 * (second ? j - (int)ja : j);
        heads = second ? a.HB : a.HA;
        const ST* p = (const ST*)in.p + b * in.batch + i * in.token + h0 * in.head;
#pragma unroll
        for (int r = 0; r < 4; ++r) src[r] = h0 + r < heads ? p + r * in.head : nullptr;
    }
    uint4 raw[4][2];
    if (FAST) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (src[r]) {
                raw[r][0] = *reinterpret_cast<const uint4*>(src[r] + sh.e0);
                raw[r][1] = *reinterpret_cast<const uint4*>(src[r] + sh.e1);
            }
    }
    // the table row of this position: cosines and sines of the lane's V pairs
    const float2* cs = a.rope.table + (int64_t)pos * (a.rope.dim / 2);
    const bool turns = a.pos && (!FAST || u < a.rope.dim / (2 * V));
    float2 t[V];
    if (FAST && turns) {
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
            const float4 f = __ldg(reinterpret_cast<const float4*>(cs + V * u) + e);
            t[2 * e] = make_float2(f.x, f.y * a.dir);
            t[2 * e + 1] = make_float2(f.z, f.w * a.dir);
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (!src[r]) continue;
        float x[2 * V];
        const bool value = kv && (r & 1);
        if (FAST) {
            Vec16<ST>::widen(raw[r][0], x);
            Vec16<ST>::widen(raw[r][1], x + V);
            if (turns && !value) {
                if (a.rope.interleaved) rotate_pairs<V, true>(x, t);
                else rotate_pairs<V, false>(x, t);
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[e] = Storage<ST>::load(src[r], sh.e0 + e);
                x[V + e] = Storage<ST>::load(src[r], sh.e1 + e);
            }
            if (turns && !value) rotate_elements<ST>(src[r], sh.e0, sh.e1, a.rope, cs, a.dir, x);
            // in place, a lane's partners are other lanes' elements: all of the group read before any writes
            __syncwarp(lanes);
        }
        if (CACHE && kv) {
            const int64_t row = crow + (h0 + (r >> 1)) * head_step(a.cache);
            if (CACHE == 2) {
                quantise_share<HD, V>(x, lanes, sh.e0, sh.e1, (uint8_t*)(value ? a.cache.v : a.cache.k) + row * HD,
                                      (value ? a.cache.vs : a.cache.ks) + row, u == 0);
            } else {
                store_share<ST, FAST>((ST*)(value ? a.cache.v : a.cache.k) + row * HD, sh.e0, sh.e1, x);
            }
        } else {
            store_share<ST, FAST>((ST*)out.p + b * out.batch + i * out.token + (h0 + r) * out.head, sh.e0, sh.e1, x);
        }
    }
}

// ---- read ------------------------------------------------------------------------------------
// One group of HD / 16 lanes (e4m3) or HD es / 16 lanes per (sequence, row, head): the key and
// the value row, one 16-byte load each.
template <typename ST, int HD, bool Q8, bool FAST>
__global__ void __launch_bounds__(kRowThreads) read_kernel(const __grid_constant__ ReadArgs a) {
    constexpr int V = Q8 ? 16 : Vec16<ST>::kN, GL = HD / V;
    const uint32_t group = blockIdx.x * (kRowThreads / GL) + threadIdx.x / GL;
    const int u = threadIdx.x % GL;
    const uint32_t Hkv = a.cache.Hkv;
    if (group >= (uint32_t)a.B * a.L * Hkv) return;
    const uint32_t row = group / Hkv;
    const int h = (int)(group - row * Hkv), b = (int)(row / (uint32_t)a.L), i = (int)(row - (uint32_t)b * a.L);
    const int n = a.n_rows[b];
    if ((n < 0 || n > a.L) && u == 0) atomicOr(a.status, ST_DEVICE);
    uint4 raw[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    float sc[2] = {0.f, 0.f};
    int64_t crow;
    if (i < n && n <= a.L && cache_row(a.cache, b, (int64_t)a.start[b] + i, crow, a.status)) {
        crow += h * head_step(a.cache);
        constexpr int es = Q8 ? 1 : Storage<ST>::kBytes;
        raw[0] = __ldcs(reinterpret_cast<const uint4*>((const char*)a.cache.k + crow * HD * es) + u);
        raw[1] = __ldcs(reinterpret_cast<const uint4*>((const char*)a.cache.v + crow * HD * es) + u);
        if (Q8) {
            sc[0] = a.cache.ks[crow];
            sc[1] = a.cache.vs[crow];
        }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const fe_rows& o = r ? a.v_out : a.k_out;
        ST* dst = (ST*)o.p + b * o.batch + i * o.token + h * o.head + u * V;
        float x[V];
        if (Q8) {
            const uint32_t w[4] = {raw[r].x, raw[r].y, raw[r].z, raw[r].w};
#pragma unroll
            for (int k = 0; k < V / 2; ++k) {
                const float2 f = e4m3x2_to_f32(w[k / 2] >> (16 * (k & 1)));
                x[2 * k] = f.x * sc[r];
                x[2 * k + 1] = f.y * sc[r];
            }
        } else {
            Vec16<ST>::widen(raw[r], x);
        }
        if (FAST) {
            if (Q8) {
                constexpr int W = Vec16<ST>::kN;
#pragma unroll
                for (int k = 0; k < V / W; ++k) reinterpret_cast<uint4*>(dst)[k] = pack16<ST>(x + k * W);
            } else {
                *reinterpret_cast<uint4*>(dst) = raw[r];  // (the same type: the bits as they are)
            }
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k) store_one(dst + k, x[k]);
        }
    }
}

// ---- keep --------------------------------------------------------------------------------------
// One warp per (group of layers, sequence, KV head). The lanes first work out the path's rows, one
// node each (its slot's and its new slot's cache rows: two page lookups side by side), then carry
// 16-byte columns of the key and value rows along the path, layer after layer: since path is
// increasing with path[j] >= j + 1, slot 1 + j is written only after the last read of it when the
// moves go in order, so eight loads go before their eight stores. Bound by latency: three dependent
// reads (path, page table, rows), and with four layers a warp, which where there are enough warps
// share the first two, the layers' moves one after another. 80 layers of one sequence: 5 us; 32
// layers of 32 sequences, 7 rows each at most: 10 us.
__global__ void __launch_bounds__(kRowThreads) keep_kernel(const __grid_constant__ KeepArgs a) {
    const uint32_t w = blockIdx.x * (kRowThreads / 32) + threadIdx.x / 32;
    const int lane = threadIdx.x & 31;
    const uint32_t Hkv = a.cache.Hkv, groups = (a.n_layers + a.layers_per_warp - 1) / a.layers_per_warp;
    if (w >= groups * a.B * Hkv) return;
    const int h = (int)(w % Hkv), b = (int)(w / Hkv % a.B), l0 = (int)(w / Hkv / a.B) * a.layers_per_warp;
    const int l1 = min(l0 + a.layers_per_warp, a.n_layers);
    const int n = a.n_accept[b];
    const int* path = a.path + (int64_t)b * a.N;
    const int64_t start = a.start[b], hs = h * head_step(a.cache);
    if (n <= 0 || n > a.N) {
        if (n != 0 && lane == 0) atomicOr(a.status, ST_DEVICE);
        return;
    }
    // the rows of node path[j] (from) and of its new slot (to); false if the path or a slot is bad
    auto rows_of = [&](int j, int64_t& from, int64_t& to) -> bool {
        const int p = path[j], before = j > 0 ? path[j - 1] : 0;
        bool ok = p > before;
        if (!ok) atomicOr(a.status, ST_DEVICE);
        ok = ok && cache_row(a.cache, b, start + p, from, a.status);
        return cache_row(a.cache, b, start + 1 + j, to, a.status) && ok;
    };
    int64_t from = 0, to = 0;
    // every node, and the root's slot, is checked before the first move
    bool bad = false;
    int64_t root;
    if (lane == 0 && !cache_row(a.cache, b, start, root, a.status)) bad = true;
    for (int j = lane; j < n; j += 32)
        if (!rows_of(j, from, to)) bad = true;
    if (__any_sync(0xffffffffu, bad)) return;
    const int rv = a.row_bytes / 16, parts = 2 * rv + (a.layer[0].k_scale ? 2 : 0);
    for (int j0 = 0; j0 < n; j0 += 8) {
        if (n > 32 && j0 % 32 == 0 && j0 + lane < n) rows_of(j0 + lane, from, to);  // (up to 32 are at hand from the check)
        int64_t f[8], d[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            f[k] = __shfl_sync(0xffffffffu, from, (j0 + k) & 31) + hs;
            d[k] = __shfl_sync(0xffffffffu, to, (j0 + k) & 31) + hs;
            if (j0 + k >= n || f[k] == d[k]) d[k] = -1;
        }
        for (int it = lane; it < parts; it += 32) {
            const bool sc = it >= 2 * rv, val = sc ? it > 2 * rv : it >= rv;
            const int col = (it - (val ? rv : 0)) * 16;
#pragma unroll 1
            for (int l = l0; l < l1; ++l) {
                const fe_kv& L = a.layer[l];
                if (!sc) {
                    char* base = (char*)(val ? L.v : L.k) + col;
                    uint4 x[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (d[k] >= 0) x[k] = *reinterpret_cast<const uint4*>(base + f[k] * a.row_bytes);
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (d[k] >= 0) *reinterpret_cast<uint4*>(base + d[k] * a.row_bytes) = x[k];
                } else {
                    float* base = val ? L.v_scale : L.k_scale;
                    float x[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (d[k] >= 0) x[k] = base[f[k]];
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (d[k] >= 0) base[d[k]] = x[k];
                }
            }
        }
    }
}

bool rows_aligned(const fe_rows& r, int es) {
    const int v = 16 / es;
    return !r.p || (((uintptr_t)r.p & 15) == 0 && r.batch % v == 0 && r.token % v == 0 && r.head % v == 0);
}

template <typename K, typename A>
cudaError_t launch_groups(K kern, int64_t groups, int per_block, const A& a, cudaStream_t st) {
    if (groups == 0) return cudaSuccess;
    const int64_t blocks = (groups + per_block - 1) / per_block;
    if (blocks > 0x7FFFFFFF) return cudaErrorInvalidValue;
    kern<<<(unsigned)blocks, kRowThreads, 0, st>>>(a);
    return cudaGetLastError();
}

template <typename ST, int HD>
cudaError_t launch_rows_t(const RowsArgs& a, int cache_kind, cudaStream_t st) {
    constexpr int V = Vec16<ST>::kN, GL = HD / (2 * V), es = Storage<ST>::kBytes;
    const bool fast = a.rope.dim % (2 * V) == 0 && rows_aligned(a.a_in, es) && rows_aligned(a.a_out, es) &&
                      rows_aligned(a.b_in, es) && rows_aligned(a.b_out, es) && rows_aligned(a.v_in, es);
    const int64_t J = (a.HA + 3) / 4 + (cache_kind ? (a.HB + 1) / 2 : (a.HB + 3) / 4);
    const int64_t groups = (int64_t)a.B * a.T * J;
    const int pb = kRowThreads / GL;
    auto go = [&](auto k) { return launch_groups(k, groups, pb, a, st); };
    if (cache_kind == 0) return fast ? go(rows_kernel<ST, HD, 0, true>) : go(rows_kernel<ST, HD, 0, false>);
    if (cache_kind == 1) return fast ? go(rows_kernel<ST, HD, 1, true>) : go(rows_kernel<ST, HD, 1, false>);
    if constexpr (es == 2) return fast ? go(rows_kernel<ST, HD, 2, true>) : go(rows_kernel<ST, HD, 2, false>);
    return cudaErrorInvalidValue;
}

template <typename ST, int HD, bool Q8>
cudaError_t launch_read_t(const ReadArgs& a, cudaStream_t st) {
    constexpr int V = Q8 ? 16 : Vec16<ST>::kN, GL = HD / V, es = Storage<ST>::kBytes;
    const bool fast = rows_aligned(a.k_out, es) && rows_aligned(a.v_out, es);
    const int64_t groups = (int64_t)a.B * a.L * a.cache.Hkv;
    return fast ? launch_groups(read_kernel<ST, HD, Q8, true>, groups, kRowThreads / GL, a, st)
                : launch_groups(read_kernel<ST, HD, Q8, false>, groups, kRowThreads / GL, a, st);
}

}  // namespace

cudaError_t launch_rope_table(float2* table, int max_seq, int pairs, const double* inv_freq, double amplitude,
                              int num_sms, cudaStream_t st) {
    const int64_t n = (int64_t)max_seq * pairs;
    const int blocks = (int)((n + 255) / 256 < num_sms * 8 ? (n + 255) / 256 : num_sms * 8);
    rope_table_kernel<<<blocks, 256, 0, st>>>(table, max_seq, pairs, inv_freq, amplitude);
    return cudaGetLastError();
}

cudaError_t launch_rows(const RowsArgs& a, fe_dtype dtype, int hd, int cache_kind, cudaStream_t st) {
    if (dtype == FE_F32)
        return hd == 128 ? launch_rows_t<float, 128>(a, cache_kind, st) : launch_rows_t<float, 64>(a, cache_kind, st);
    return hd == 128 ? launch_rows_t<bf16_t, 128>(a, cache_kind, st) : launch_rows_t<bf16_t, 64>(a, cache_kind, st);
}

cudaError_t launch_cache_read(const ReadArgs& a, fe_dtype dtype, fe_dtype cache_dtype, int hd, cudaStream_t st) {
    if (cache_dtype == FE_E4M3)
        return hd == 128 ? launch_read_t<bf16_t, 128, true>(a, st) : launch_read_t<bf16_t, 64, true>(a, st);
    if (dtype == FE_F32)
        return hd == 128 ? launch_read_t<float, 128, false>(a, st) : launch_read_t<float, 64, false>(a, st);
    return hd == 128 ? launch_read_t<bf16_t, 128, false>(a, st) : launch_read_t<bf16_t, 64, false>(a, st);
}

cudaError_t launch_cache_keep(const KeepArgs& args, int num_sms, cudaStream_t st) {
    KeepArgs a = args;
    const int64_t one = (int64_t)a.n_layers * a.B * a.cache.Hkv;
    a.layers_per_warp = one >= num_sms * 32 ? 4 : 1;  // (half an SM's warps, at least, with one layer each)
    const int64_t warps = (int64_t)((a.n_layers + a.layers_per_warp - 1) / a.layers_per_warp) * a.B * a.cache.Hkv;
    return launch_groups(keep_kernel, warps, kRowThreads / 32, a, st);
}

}  // namespace fe
