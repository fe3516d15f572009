// C ABI of the target-side operators (include/fe_target.h): the handle (rotation table,
// attention workspace, status word) and the argument checks of each call.
#include <math.h>
#include <stdio.h>

#include <new>
#include <vector>

#include "fe_target_kernels.h"

using namespace fe;

struct fe_target {
    fe_target_config cfg;
    int device = 0, num_sms = 0;
    float2* rope = nullptr;
    float *part_o = nullptr, *part_ml = nullptr;
    int* status = nullptr;
    SplitDesc* split = nullptr;
};

namespace {

fe_status fail(cudaError_t e, const char* what) {
    char buf[200];
    snprintf(buf, sizeof(buf), "%s (fe_target.cu): %s", what, cudaGetErrorString(e));
    set_error_detail(buf);
    return e == cudaErrorMemoryAllocation ? FE_ERR_OOM : FE_ERR_CUDA;
}

#define FE_TRY(call)                                   \
    do {                                               \
        cudaError_t _e = (call);                       \
        if (_e != cudaSuccess) return fail(_e, #call); \
    } while (0)

fe_status check_device(const fe_target* t) {
    int dev = -1;
    FE_TRY(cudaGetDevice(&dev));
    if (dev == t->device) return FE_OK;
    char buf[128];
    snprintf(buf, sizeof(buf), "the current CUDA device (%d) is not the handle's device (%d)", dev, t->device);
    set_error_detail(buf);
    return FE_ERR_INVALID_ARG;
}

bool valid_config(const fe_target_config* c) {
    if (!c) return false;
    if (c->n_heads < 1 || c->n_kv_heads < 1 || c->n_heads % c->n_kv_heads) return false;
    if (c->max_batch < 1 || c->max_batch > 65535 || c->max_seq < 1 || c->max_seq > (1 << 28) || c->page_size < 0) return false;
    if (c->head_dim < 1) return false;
    if (c->dtype != FE_F32 && c->dtype != FE_BF16) return false;
    if (c->cache_dtype != FE_F32 && c->cache_dtype != FE_BF16 && c->cache_dtype != FE_E4M3) return false;
    if (c->rope_dim < 2 || c->rope_dim % 2 || c->rope_dim > c->head_dim) return false;
    if (c->rope_layout != FE_ROPE_HALF && c->rope_layout != FE_ROPE_INTERLEAVED) return false;
    if (!(c->rope_theta > 1.f) || isinf(c->rope_theta)) return false;
    const int k = c->rope_scaling;
    if (k < FE_ROPE_NONE || k > FE_ROPE_YARN) return false;
    if (k != FE_ROPE_NONE && (!(c->rope_factor >= 1.f) || isinf(c->rope_factor))) return false;
    if (k == FE_ROPE_NTK && c->rope_dim <= 2) return false;
    if (k == FE_ROPE_BANDS || k == FE_ROPE_YARN) {
        if (!(c->rope_orig >= 1.f) || isinf(c->rope_orig) || isinf(c->rope_low) || isinf(c->rope_high)) return false;
        const float lo = k == FE_ROPE_BANDS ? c->rope_low : c->rope_high, hi = k == FE_ROPE_BANDS ? c->rope_high : c->rope_low;
        if (!(lo > 0.f) || !(hi > lo)) return false;
    }
    return true;
}

bool supported_config(const fe_target_config* c) {
    if (c->head_dim != 64 && c->head_dim != 128) return false;
    return c->cache_dtype == c->dtype || (c->dtype == FE_BF16 && c->cache_dtype == FE_E4M3);
}

// frequencies (radians per position) of the rotated pairs, and the amplitude of cos and sin
std::vector<double> rope_freqs(const fe_target_config& c, double* amplitude) {
    const int rd = c.rope_dim;
    const double theta = c.rope_theta, s = c.rope_factor, L = c.rope_orig, pi2 = 6.283185307179586;
    std::vector<double> f(rd / 2);
    *amplitude = 1.0;
    double lo = 0.0, hi = 0.0;
    if (c.rope_scaling == FE_ROPE_YARN) {
        const auto dim = [&](double turns) { return rd * log(L / (turns * pi2)) / (2.0 * log(theta)); };
        lo = fmax(floor(dim(c.rope_low)), 0.0);
        hi = fmin(ceil(dim(c.rope_high)), rd - 1.0);
        *amplitude = 0.1 * log(s) + 1.0;
    }
    for (int i = 0; i < rd / 2; ++i) {
        const double e = -2.0 * i / rd, b = pow(theta, e);
        switch (c.rope_scaling) {
            case FE_ROPE_LINEAR: f[i] = b / s; break;
            case FE_ROPE_NTK: f[i] = pow(theta * pow(s, rd / (rd - 2.0)), e); break;
            case FE_ROPE_BANDS: {
                const double w = fmin(fmax((L * b / pi2 - c.rope_low) / ((double)c.rope_high - c.rope_low), 0.0), 1.0);
                f[i] = b * ((1.0 - w) / s + w);
                break;
            }
            case FE_ROPE_YARN: {
                const double w = fmin(fmax((i - lo) / fmax(hi - lo, 0.001), 0.0), 1.0);
                f[i] = b * (w / s + 1.0 - w);
                break;
            }
            default: f[i] = b;
        }
    }
    return f;
}

void release(fe_target* t) {
    cudaFree(t->rope);
    cudaFree(t->part_o);
    cudaFree(t->part_ml);
    cudaFree(t->status);
    cudaFree(t->split);
    delete t;
}

fe_status build(fe_target* t, cudaStream_t st) {
    const fe_target_config& c = t->cfg;
    FE_TRY(cudaGetDevice(&t->device));
    FE_TRY(cudaDeviceGetAttribute(&t->num_sms, cudaDevAttrMultiProcessorCount, t->device));
    FE_TRY(tree_attn_prepare());
    const int pairs = c.rope_dim / 2;
    const size_t rows = (size_t)t->num_sms * 2 * kAttnItemRows;
    FE_TRY(cudaMalloc((void**)&t->rope, (size_t)c.max_seq * pairs * sizeof(float2)));
    FE_TRY(cudaMalloc((void**)&t->part_o, rows * c.head_dim * sizeof(float)));
    FE_TRY(cudaMalloc((void**)&t->part_ml, rows * 2 * sizeof(float)));
    FE_TRY(cudaMalloc((void**)&t->status, sizeof(int)));
    FE_TRY(cudaMalloc((void**)&t->split, (size_t)t->num_sms * kAttnCtasPerSm * sizeof(SplitDesc)));
    FE_TRY(cudaMemsetAsync(t->status, 0, sizeof(int), st));
    FE_TRY(cudaMemsetAsync(t->split, 0, (size_t)t->num_sms * kAttnCtasPerSm * sizeof(SplitDesc), st));
    double amplitude = 1.0;
    const std::vector<double> f = rope_freqs(c, &amplitude);
    double* df = nullptr;
    FE_TRY(cudaMalloc((void**)&df, f.size() * sizeof(double)));
    cudaError_t e = cudaMemcpyAsync(df, f.data(), f.size() * sizeof(double), cudaMemcpyHostToDevice, st);
    if (e == cudaSuccess) e = launch_rope_table(t->rope, c.max_seq, pairs, df, amplitude, t->num_sms, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    cudaFree(df);
    FE_TRY(e);
    return FE_OK;
}

bool kv_ok(const fe_target* t, const fe_kv& kv) {
    if (!kv.k || !kv.v || ((uintptr_t)kv.k & 15) || ((uintptr_t)kv.v & 15)) return false;
    return t->cfg.cache_dtype != FE_E4M3 || (kv.k_scale && kv.v_scale);
}

bool pages_ok(const fe_target* t, const fe_pages& p) { return t->cfg.page_size == 0 || (p.table && p.n_pages >= 1); }

bool shape_ok(const fe_target* t, int B, int T) {
    return B >= 1 && B <= t->cfg.max_batch && T >= 1 && T <= t->cfg.max_seq &&
           (int64_t)B * T * (t->cfg.n_heads + t->cfg.n_kv_heads) <= 1 << 30;
}

CacheView cache_view(const fe_target* t, const fe_kv& kv, const fe_pages& p) {
    const fe_target_config& c = t->cfg;
    CacheView v{};
    v.k = kv.k;
    v.v = kv.v;
    v.ks = kv.k_scale;
    v.vs = kv.v_scale;
    v.table = p.table;
    v.n_pages = p.n_pages;
    v.page_size = c.page_size;
    v.max_pages = c.page_size ? (c.max_seq + c.page_size - 1) / c.page_size : 0;
    v.max_seq = c.max_seq;
    v.Hkv = c.n_kv_heads;
    return v;
}

RowsArgs rows_args(const fe_target* t) {
    RowsArgs r{};
    r.rope = RopeView{t->rope, t->cfg.rope_dim, t->cfg.rope_layout == FE_ROPE_INTERLEAVED, t->cfg.max_seq};
    r.dir = 1.f;
    r.status = t->status;
    return r;
}

bool rows_on(int bytes, const fe_rows& r, int es) {
    const int v = bytes / es;
    return ((uintptr_t)r.p & (bytes - 1)) == 0 && r.batch % v == 0 && r.token % v == 0 && r.head % v == 0;
}

}  // namespace

extern "C" {

fe_status fe_target_init(const fe_target_config* cfg, void* stream, fe_target** out) {
    if (!out) return FE_ERR_INVALID_ARG;
    *out = nullptr;
    if (!valid_config(cfg)) return FE_ERR_INVALID_ARG;
    if (!supported_config(cfg)) return FE_ERR_UNSUPPORTED;
    fe_target* t = new (std::nothrow) fe_target();
    if (!t) return FE_ERR_OOM;
    t->cfg = *cfg;
    fe_status rc;
    try {
        rc = build(t, (cudaStream_t)stream);
    } catch (...) {
        rc = FE_ERR_OOM;
    }
    if (rc != FE_OK) {
        release(t);
        return rc;
    }
    *out = t;
    return FE_OK;
}

void fe_target_free(fe_target* t) {
    if (!t) return;
    int cur = -1;
    const bool have = cudaGetDevice(&cur) == cudaSuccess;
    const int dev = t->device;
    if (have && cur != dev) cudaSetDevice(dev);
    cudaDeviceSynchronize();
    release(t);
    if (have && cur != dev) cudaSetDevice(cur);
}

fe_status fe_target_status(fe_target* t, void* stream) {
    if (!t) return FE_ERR_INVALID_ARG;
    const fe_status dv = check_device(t);
    if (dv != FE_OK) return dv;
    cudaStream_t st = (cudaStream_t)stream;
    // (on `st` itself: the default stream is not ordered with it, so that a clear there could come after
    // the next call's errors, and it may have long work of others queued)
    int v = 0;
    FE_TRY(cudaMemcpyAsync(&v, t->status, sizeof(int), cudaMemcpyDeviceToHost, st));
    FE_TRY(cudaMemsetAsync(t->status, 0, sizeof(int), st));
    FE_TRY(cudaStreamSynchronize(st));
    if (v & ST_TIMEOUT) return FE_ERR_TIMEOUT;
    if (v & ST_CAPACITY) return FE_ERR_CAPACITY;
    if (v & ST_DEVICE) return FE_ERR_DEVICE;
    return FE_OK;
}

fe_status fe_rope(fe_target* t, const fe_rope_args* a, void* stream) {
    if (!t || !a || !a->pos || (!a->q.p && !a->k.p)) return FE_ERR_INVALID_ARG;
    if ((a->q.p && !a->q_out.p) || (a->k.p && !a->k_out.p) || !shape_ok(t, a->B, a->T)) return FE_ERR_INVALID_ARG;
    const fe_status dv = check_device(t);
    if (dv != FE_OK) return dv;
    RowsArgs r = rows_args(t);
    r.B = a->B;
    r.T = a->T;
    r.pos = a->pos;
    r.dir = a->backward ? -1.f : 1.f;
    if (a->q.p) {
        r.HA = t->cfg.n_heads;
        r.a_in = a->q;
        r.a_out = a->q_out;
    }
    if (a->k.p) {
        r.HB = t->cfg.n_kv_heads;
        r.b_in = a->k;
        r.b_out = a->k_out;
    }
    FE_TRY(launch_rows(r, t->cfg.dtype, t->cfg.head_dim, 0, (cudaStream_t)stream));
    return FE_OK;
}

fe_status fe_cache_write(fe_target* t, const fe_cache_write_args* a, void* stream) {
    if (!t || !a || !a->k.p || !a->v.p || !a->start || !shape_ok(t, a->B, a->T)) return FE_ERR_INVALID_ARG;
    if (a->q.p && (!a->q_out.p || !a->pos)) return FE_ERR_INVALID_ARG;
    if (!kv_ok(t, a->cache) || !pages_ok(t, a->pages)) return FE_ERR_INVALID_ARG;
    const fe_status dv = check_device(t);
    if (dv != FE_OK) return dv;
    RowsArgs r = rows_args(t);
    r.B = a->B;
    r.T = a->T;
    r.pos = a->pos;
    r.start = a->start;
    r.n_rows = a->n_rows;
    if (a->q.p) {
        r.HA = t->cfg.n_heads;
        r.a_in = a->q;
        r.a_out = a->q_out;
    }
    r.HB = t->cfg.n_kv_heads;
    r.b_in = a->k;
    r.v_in = a->v;
    r.cache = cache_view(t, a->cache, a->pages);
    FE_TRY(launch_rows(r, t->cfg.dtype, t->cfg.head_dim, t->cfg.cache_dtype == FE_E4M3 ? 2 : 1, (cudaStream_t)stream));
    return FE_OK;
}

fe_status fe_cache_read(fe_target* t, const fe_cache_read_args* a, void* stream) {
    if (!t || !a || !a->start || !a->n_rows || !a->k_out.p || !a->v_out.p || !shape_ok(t, a->B, a->L))
        return FE_ERR_INVALID_ARG;
    if (!kv_ok(t, a->cache) || !pages_ok(t, a->pages)) return FE_ERR_INVALID_ARG;
    const fe_status dv = check_device(t);
    if (dv != FE_OK) return dv;
    ReadArgs r{};
    r.B = a->B;
    r.L = a->L;
    r.start = a->start;
    r.n_rows = a->n_rows;
    r.cache = cache_view(t, a->cache, a->pages);
    r.k_out = a->k_out;
    r.v_out = a->v_out;
    r.status = t->status;
    FE_TRY(launch_cache_read(r, t->cfg.dtype, t->cfg.cache_dtype, t->cfg.head_dim, (cudaStream_t)stream));
    return FE_OK;
}

fe_status fe_tree_attention(fe_target* t, const fe_tree_attention_args* a, void* stream) {
    if (!t || !a || !a->q.p || !a->out.p || !a->prefix_len || !shape_ok(t, a->B, a->T)) return FE_ERR_INVALID_ARG;
    if (!kv_ok(t, a->cache) || !pages_ok(t, a->pages) || !isfinite(a->scale) || a->scale <= 0.f)
        return FE_ERR_INVALID_ARG;
    const fe_status dv = check_device(t);
    if (dv != FE_OK) return dv;
    const fe_target_config& c = t->cfg;
    const int es = c.dtype == FE_F32 ? 4 : 2;
    TreeAttnArgs r{};
    r.B = a->B;
    r.T = a->T;
    r.H = c.n_heads;
    r.Hkv = c.n_kv_heads;
    r.G = c.n_heads / c.n_kv_heads;
    r.q = a->q;
    r.out = a->out;
    r.lse = a->lse;
    r.prefix = a->prefix_len;
    r.nodes = a->n_nodes;
    r.mask = a->mask;
    r.scale = a->scale;
    r.cache = cache_view(t, a->cache, a->pages);
    r.split = t->split;
    r.part_o = t->part_o;
    r.part_ml = t->part_ml;
    r.status = t->status;
    r.q_vec = rows_on(16, a->q, es);
    r.out_vec = rows_on(32, a->out, es) ? 2 : rows_on(16, a->out, es);
    if (!tree_attn_fits(r, c.dtype, c.cache_dtype)) return FE_ERR_UNSUPPORTED;
    FE_TRY(launch_tree_attn(r, c.dtype, c.cache_dtype, c.head_dim, t->num_sms, (cudaStream_t)stream));
    return FE_OK;
}

fe_status fe_cache_keep(fe_target* t, const fe_cache_keep_args* a, void* stream) {
    if (!t || !a || !a->path || !a->n_accept || !a->start || !a->caches) return FE_ERR_INVALID_ARG;
    if (a->B < 1 || a->B > t->cfg.max_batch || a->N < 1 || a->N > t->cfg.max_seq || a->n_layers < 1)
        return FE_ERR_INVALID_ARG;
    for (int i = 0; i < a->n_layers; ++i)
        if (!kv_ok(t, a->caches[i])) return FE_ERR_INVALID_ARG;
    if (!pages_ok(t, a->pages)) return FE_ERR_INVALID_ARG;
    const fe_status dv = check_device(t);
    if (dv != FE_OK) return dv;
    const fe_target_config& c = t->cfg;
    KeepArgs r{};
    r.B = a->B;
    r.N = a->N;
    r.row_bytes = c.head_dim * (c.cache_dtype == FE_F32 ? 4 : c.cache_dtype == FE_BF16 ? 2 : 1);
    r.path = a->path;
    r.n_accept = a->n_accept;
    r.start = a->start;
    r.cache = cache_view(t, fe_kv{}, a->pages);
    r.status = t->status;
    for (int l0 = 0; l0 < a->n_layers; l0 += kKeepMaxLayers) {
        r.n_layers = a->n_layers - l0 < kKeepMaxLayers ? a->n_layers - l0 : kKeepMaxLayers;
        for (int i = 0; i < r.n_layers; ++i) {
            r.layer[i] = a->caches[l0 + i];
            if (c.cache_dtype != FE_E4M3) r.layer[i].k_scale = r.layer[i].v_scale = nullptr;
        }
        FE_TRY(launch_cache_keep(r, t->num_sms, (cudaStream_t)stream));
    }
    return FE_OK;
}

}  // extern "C"
