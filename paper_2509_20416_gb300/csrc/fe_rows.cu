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

template <typename ST, bool FAST>
__device__ __forceinline__ void load_share(const ST* row, int e0, int e1, float* x) {
    constexpr int V = Vec16<ST>::kN;
    if (FAST) {
        const uint4 a = *reinterpret_cast<const uint4*>(row + e0), b = *reinterpret_cast<const uint4*>(row + e1);
        Vec16<ST>::widen(a, x);
        Vec16<ST>::widen(b, x + V);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            x[j] = Storage<ST>::load(row, e0 + j);
            x[V + j] = Storage<ST>::load(row, e1 + j);
        }
    }
}

// Rotate a lane's elements x (loaded from `row`) to the position whose table row is `cs`.
template <typename ST, bool FAST>
__device__ __forceinline__ void rotate_share(const ST* row, int u, int e0, int e1, const RopeView& r, const float2* cs,
                                             float dir, float* x) {
    constexpr int V = Vec16<ST>::kN;
    if (FAST) {
        if (u >= r.dim / (2 * V)) return;
        float2 t[V];
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            const float4 f = __ldg(reinterpret_cast<const float4*>(cs + V * u) + j);
            t[2 * j] = make_float2(f.x, f.y * dir);
            t[2 * j + 1] = make_float2(f.z, f.w * dir);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {  // pair j of this unit: (x[j], x[V + j]), or neighbours
            const int ia = r.interleaved ? 2 * j : j, ib = r.interleaved ? 2 * j + 1 : V + j;
            float& a = x[ia];
            float& b = x[ib];
            const float ya = a * t[j].x - b * t[j].y, yb = b * t[j].x + a * t[j].y;
            a = ya;
            b = yb;
        }
    } else {
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

// One group per job: a token's two rotated heads (2 j, 2 j + 1), or a KV head's key and value
// rows. Two rows a lane keep 64 bytes in flight, and a key and its value share one address.
template <typename ST, int HD, int CACHE, bool FAST>
__global__ void __launch_bounds__(kRowThreads) rows_kernel(const RowsArgs a) {
    constexpr int V = Vec16<ST>::kN, GL = HD / (2 * V);
    const int ja = (a.HA + 1) / 2, jb = CACHE ? a.HB : (a.HB + 1) / 2, J = ja + jb;
    const int64_t group = (int64_t)blockIdx.x * (kRowThreads / GL) + threadIdx.x / GL;
    const int u = threadIdx.x % GL;
    const bool live = group < (int64_t)a.B * a.T * J;
    const int64_t token = live ? group / J : 0;
    const int j = (int)(group - token * J), b = (int)(token / a.T), i = (int)(token - (int64_t)b * a.T);
    const Share<V> sh(u, a.rope);
    // the group's lanes of the warp: they take every branch below together
    const unsigned lanes = ((1u << GL) - 1u) << ((threadIdx.x & 31) / GL * GL);

    const bool kv = CACHE && live && j >= ja;
    const ST* src[2] = {nullptr, nullptr};
    ST* dst[2] = {nullptr, nullptr};
    bool rot[2] = {true, true};
    int64_t crow = 0;
    if (live) {
        int pos = 0;
        bool pos_ok = true;
        if (a.pos) {
            pos = a.pos[token];
            pos_ok = pos >= 0 && pos < a.rope.max_pos;
            if (!pos_ok && u == 0) atomicOr(a.status, ST_CAPACITY);
        } else {
            rot[0] = false;
        }
        if (kv) {
            const int h = j - ja;
            const int n = a.n_rows ? a.n_rows[b] : a.T;
            if ((n < 0 || n > a.T) && u == 0) atomicOr(a.status, ST_DEVICE);
            rot[1] = false;
            if (pos_ok && i < n && n <= a.T && cache_row(a.cache, b, (int64_t)a.start[b] + i, crow, a.status)) {
                crow += h * head_step(a.cache);
                src[0] = (const ST*)a.b_in.p + b * a.b_in.batch + i * a.b_in.token + h * a.b_in.head;
                src[1] = (const ST*)a.v_in.p + b * a.v_in.batch + i * a.v_in.token + h * a.v_in.head;
                if (CACHE == 1) {
                    dst[0] = (ST*)a.cache.k + crow * HD;
                    dst[1] = (ST*)a.cache.v + crow * HD;
                }
            }
        } else if (pos_ok) {
            const bool second = !CACHE && j >= ja;
            const fe_rows &in = second ? a.b_in : a.a_in, &out = second ? a.b_out : a.a_out;
            const int heads = second ? a.HB : a.HA;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int h = 2 * (second ? j - ja : j) + r;
                if (h >= heads) continue;
                src[r] = (const ST*)in.p + b * in.batch + i * in.token + h * in.head;
                dst[r] = (ST*)out.p + b * out.batch + i * out.token + h * out.head;
            }
        }
        // (the table row of a skipped position is never read: src stays null)
        const float2* cs = a.rope.table + (int64_t)pos * (a.rope.dim / 2);
        float x[2][2 * V];
#pragma unroll
        for (int r = 0; r < 2; ++r)
            if (src[r]) load_share<ST, FAST>(src[r], sh.e0, sh.e1, x[r]);
#pragma unroll
        for (int r = 0; r < 2; ++r)
            if (src[r] && rot[r]) rotate_share<ST, FAST>(src[r], u, sh.e0, sh.e1, a.rope, cs, a.dir, x[r]);
        if (CACHE == 2 && kv) {
            // (src is set for both rows or none, alike in the group's lanes)
            if (src[0]) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float m = 0.f;
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) m = fmaxf(m, finite_f32(x[r][e]) ? fabsf(x[r][e]) : 0.f);
#pragma unroll
                    for (int o = GL / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(lanes, m, o));
                    const int c = scale_exp(m);
                    const float inv = pow2(-c);
                    uint8_t* out = (uint8_t*)(r ? a.cache.v : a.cache.k) + crow * HD;
                    uint32_t w[V / 2];
#pragma unroll
                    for (int e = 0; e < 2 * V; e += 4) {
                        float y[4];
#pragma unroll
                        for (int z = 0; z < 4; ++z)  // (a non-finite element becomes NaN)
                            y[z] = finite_f32(x[r][e + z]) ? x[r][e + z] * inv : __uint_as_float(0x7FC00000u);
                        w[e / 4] = f32x2_to_e4m3(y[0], y[1]) | (f32x2_to_e4m3(y[2], y[3]) << 16);
                    }
                    if (V == 8) {
                        *reinterpret_cast<uint2*>(out + sh.e0) = make_uint2(w[0], w[1]);
                        *reinterpret_cast<uint2*>(out + sh.e1) = make_uint2(w[V / 4], w[V / 4 + 1]);
                    } else {
                        *reinterpret_cast<uint32_t*>(out + sh.e0) = w[0];
                        *reinterpret_cast<uint32_t*>(out + sh.e1) = w[V / 4];
                    }
                    if (u == 0) (r ? a.cache.vs : a.cache.ks)[crow] = pow2(c);
                }
            }
        } else {
            // in place and element-wise, a lane's partners are other lanes' elements: all lanes
            // of the group read before any writes
            if (!FAST) __syncwarp(lanes);
#pragma unroll
            for (int r = 0; r < 2; ++r)
                if (dst[r]) store_share<ST, FAST>(dst[r], sh.e0, sh.e1, x[r]);
        }
    }
}

// ---- read ------------------------------------------------------------------------------------
// One group of HD / 16 lanes (e4m3) or HD es / 16 lanes per (sequence, row, head): the key and
// the value row, one 16-byte load each.
template <typename ST, int HD, bool Q8, bool FAST>
__global__ void __launch_bounds__(kRowThreads) read_kernel(const ReadArgs a) {
    constexpr int V = Q8 ? 16 : Vec16<ST>::kN, GL = HD / V;
    const int64_t group = (int64_t)blockIdx.x * (kRowThreads / GL) + threadIdx.x / GL;
    const int u = threadIdx.x % GL;
    const int Hkv = a.cache.Hkv;
    if (group >= (int64_t)a.B * a.L * Hkv) return;
    const int64_t row = group / Hkv;
    const int h = (int)(group - row * Hkv), b = (int)(row / a.L), i = (int)(row - (int64_t)b * a.L);
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
// One warp per (layer, sequence, KV head). A lane carries one 16-byte column of the key or value
// rows along the path: since path is increasing with path[j] >= j + 1, slot 1 + j is written only
// after the last read of it when the moves go in order, so eight loads at a time may go before
// their eight stores. Nothing crosses lanes.
__global__ void __launch_bounds__(kRowThreads) keep_kernel(const __grid_constant__ KeepArgs a) {
    const int64_t w = (int64_t)blockIdx.x * (kRowThreads / 32) + threadIdx.x / 32;
    const int lane = threadIdx.x & 31;
    const int Hkv = a.cache.Hkv;
    if (w >= (int64_t)a.n_layers * a.B * Hkv) return;
    const int h = (int)(w % Hkv);
    const int b = (int)(w / Hkv % a.B);
    const fe_kv& L = a.layer[w / Hkv / a.B];
    const int n = a.n_accept[b];
    const int* path = a.path + (int64_t)b * a.N;
    const int64_t start = a.start[b];
    if (n <= 0 || n > a.N) {
        if (n != 0 && lane == 0) atomicOr(a.status, ST_DEVICE);
        return;
    }
    // every slot and page of the path is checked before the first move
    int bad = 0;
    for (int j = lane; j <= n; j += 32) {
        int64_t row;
        if (j < n) {
            const int p = path[j];
            if (p < 1 || (j > 0 && path[j - 1] >= p)) {
                atomicOr(a.status, ST_DEVICE);
                bad = 1;
            } else if (!cache_row(a.cache, b, start + p, row, a.status)) {
                bad = 1;
            }
        }
        if (j > 0 && !cache_row(a.cache, b, start + j, row, a.status)) bad = 1;
    }
    if (__any_sync(0xffffffffu, bad)) return;
    const int64_t hs = h * head_step(a.cache);
    const int rv = a.row_bytes / 16;
    const bool scaled = L.k_scale != nullptr;
    for (int it = lane; it < 2 * rv + (scaled ? 2 : 0); it += 32) {
        const bool sc = it >= 2 * rv;
        const bool val = sc ? it > 2 * rv : it >= rv;
        char* base = (char*)(val ? L.v : L.k) + (it - (val ? rv : 0)) * 16;
        float* sbase = val ? L.v_scale : L.k_scale;
        for (int j0 = 0; j0 < n; j0 += 8) {
            uint4 x[8];
            int64_t to[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                to[k] = -1;
                if (j0 + k >= n) continue;
                int64_t from = 0;
                cache_row(a.cache, b, start + path[j0 + k], from, a.status);
                cache_row(a.cache, b, start + 1 + j0 + k, to[k], a.status);
                if (from == to[k]) {
                    to[k] = -1;
                    continue;
                }
                if (sc) x[k].x = __float_as_uint(sbase[from + hs]);
                else x[k] = *reinterpret_cast<const uint4*>(base + (from + hs) * a.row_bytes);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (to[k] < 0) continue;
                if (sc) sbase[to[k] + hs] = __uint_as_float(x[k].x);
                else *reinterpret_cast<uint4*>(base + (to[k] + hs) * a.row_bytes) = x[k];
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
    const int64_t J = (a.HA + 1) / 2 + (cache_kind ? a.HB : (a.HB + 1) / 2);
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
                              cudaStream_t st) {
    const int64_t n = (int64_t)max_seq * pairs;
    const int blocks = (int)((n + 255) / 256 < 152 * 8 ? (n + 255) / 256 : 152 * 8);
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

cudaError_t launch_cache_keep(const KeepArgs& a, cudaStream_t st) {
    const int64_t warps = (int64_t)a.n_layers * a.B * a.cache.Hkv;
    return launch_groups(keep_kernel, warps, kRowThreads / 32, a, st);
}

}  // namespace fe
