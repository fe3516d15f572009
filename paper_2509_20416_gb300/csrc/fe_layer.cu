// C ABI of the dense operators of a target layer (include/fe_layer.h): argument checks, and the
// division of a call's workspace.
#include <math.h>

#include "fe_layer_kernels.h"
#include "fe_target_handle.h"

#define FE_SOURCE "fe_layer.cu"

using namespace fe;

namespace {

constexpr int64_t kMaxRows = 1 << 30;
constexpr int kMaxCols = 1 << 24, kMaxNorm = 1 << 20;

int elem(const fe_target* t) { return t->cfg.dtype == FE_F32 ? 4 : 2; }

bool sizes_ok(int64_t M, int N, int K) { return M >= 0 && M <= kMaxRows && N >= 1 && N <= kMaxCols && K >= 1 && K <= kMaxCols; }

bool aligned_to(const void* p, int n) { return ((uintptr_t)p & (n - 1)) == 0; }

// A given matrix that is read (rows of any non-negative stride), and one that is written (rows apart).
bool in_ok(const fe_mat& m, int es) { return m.p && m.row >= 0 && aligned_to(m.p, es); }
bool out_ok(const fe_mat& m, int64_t rows, int64_t cols, int es) {
    return m.p && aligned_to(m.p, es) && m.row >= 0 && (rows <= 1 || m.row >= cols);
}
bool opt_in(const fe_mat& m, int es) { return !m.p || in_ok(m, es); }
bool opt_out(const fe_mat& m, int64_t rows, int64_t cols, int es) { return !m.p || out_ok(m, rows, cols, es); }
bool opt_ptr(const void* p, int es) { return !p || aligned_to(p, es); }

bool on16(const void* p) { return aligned_to(p, 16); }
bool on16(const fe_mat& m, int es) { return !m.p || (on16(m.p) && m.row % (16 / es) == 0); }

bool act_ok(fe_act a) { return a >= FE_ACT_NONE && a <= FE_ACT_GELU; }

// A call's workspace, handed out from its start; with a base of NULL only counted.
struct Workspace {
    char* base;
    int64_t used = 0;
    void* take(int64_t bytes) {
        char* p = base ? base + used : nullptr;
        used += (bytes + 255) / 256 * 256;
        return p;
    }
    bool fits(void* work, int64_t bytes) const { return used == 0 || (work && aligned_to(work, 256) && bytes >= used); }
};

// rows of a temporary matrix lie on 16-byte boundaries
fe_mat take_rows(Workspace& w, int64_t rows, int64_t cols, int es) {
    const int64_t row = (cols + 16 / es - 1) / (16 / es) * (16 / es);
    return fe_mat{w.take(rows * row * es), row};
}

bool project_ok(const fe_target* t, const fe_project_args* a) {
    if (!t || !a || !sizes_ok(a->M, a->N, a->K) || !act_ok(a->act)) return false;
    const int es = elem(t);
    return in_ok(a->x, es) && in_ok(a->w, es) && opt_ptr(a->bias, es) && opt_in(a->residual, es) &&
           out_ok(a->out, a->M, a->N, es) && opt_out(a->pre, a->M, a->N, 4);
}

bool project_backward_ok(const fe_target* t, const fe_project_backward_args* a) {
    if (!t || !a || !sizes_ok(a->M, a->N, a->K) || !act_ok(a->act)) return false;
    const int es = elem(t);
    if (!a->dx.p && !a->dw.p && !a->dbias) return false;
    if ((a->dx.p && !a->w.p) || (a->dw.p && !a->x.p) || (a->act != FE_ACT_NONE && !a->pre.p)) return false;
    return in_ok(a->dout, es) && opt_in(a->x, es) && opt_in(a->w, es) && opt_in(a->pre, 4) && opt_ptr(a->dbias, es) &&
           opt_out(a->dx, a->M, a->K, es) && opt_out(a->dw, a->N, a->K, es);
}

bool gated_ok(const fe_target* t, const fe_gated_ffn_args* a) {
    if (!t || !a || !sizes_ok(a->M, a->F, a->K) || !act_ok(a->act)) return false;
    const int es = elem(t);
    return in_ok(a->x, es) && in_ok(a->w_gate, es) && in_ok(a->w_up, es) && out_ok(a->out, a->M, a->F, es) &&
           !a->gate_pre.p == !a->up_pre.p && opt_out(a->gate_pre, a->M, a->F, 4) && opt_out(a->up_pre, a->M, a->F, 4);
}

bool gated_backward_ok(const fe_target* t, const fe_gated_ffn_backward_args* a) {
    if (!t || !a || !sizes_ok(a->M, a->F, a->K) || !act_ok(a->act)) return false;
    const int es = elem(t);
    if (a->w_down.p && (a->N < 1 || a->N > kMaxCols)) return false;
    if (a->dw_down.p && !a->w_down.p) return false;
    if (!a->dw_gate.p != !a->dw_up.p || (!a->dx.p && !a->dw_gate.p && !a->dw_down.p)) return false;
    if ((a->dx.p && (!a->w_gate.p || !a->w_up.p)) || (a->dw_gate.p && !a->x.p)) return false;
    return in_ok(a->dout, es) && in_ok(a->gate_pre, 4) && in_ok(a->up_pre, 4) && opt_in(a->x, es) && opt_in(a->w_gate, es) &&
           opt_in(a->w_up, es) && opt_in(a->w_down, es) && opt_out(a->dx, a->M, a->K, es) && opt_out(a->dw_gate, a->F, a->K, es) &&
           opt_out(a->dw_up, a->F, a->K, es) && opt_out(a->dw_down, a->N, a->F, es);
}

// What a call does once its arguments are checked; where its work is only counted nothing is launched
// and st is not looked at.
fe_status gemm(const fe_target* t, GemmArgs& g, Workspace& w, bool count, cudaStream_t st) {
    g.status = t->status;
    if (t->cfg.dtype == FE_F32) {
        if (!count) FE_TRY(launch_gemm_simt(g, t->num_sms, st));
        return FE_OK;
    }
    // rows off 16-byte boundaries are copied: the copy costs what the operand's bytes do, products on the
    // CUDA cores would cost some twenty times the tensor cores' time
    const auto readable = [&](fe_mat& m, int64_t rows, int64_t cols) -> fe_status {
        if (gemm_tc_reads(m, rows, cols)) return FE_OK;
        const fe_mat to = take_rows(w, rows, cols, 2);
        if (!count) FE_TRY(launch_pack_rows(m, to, rows, cols, t->num_sms, st));
        m = to;
        return FE_OK;
    };
    for (int i = 0; i < 2; ++i) {
        fe_status s = FE_OK;
        if (i == 0 || g.segs == 2 || g.twice) s = g.a_t ? readable(g.a[i], g.K, g.M) : readable(g.a[i], g.M, g.K);
        if (s == FE_OK && (i == 0 || g.segs == 2 || g.e.kind == FINISH_GATED))
            s = g.b_t ? readable(g.b[i], g.K, g.N) : readable(g.b[i], g.N, g.K);
        if (s != FE_OK) return s;
    }
    if (count) return FE_OK;
    const bool few = gemm_few_takes(g);
    const fe_status s = few ? set_up(t, GEMM_FEW, gemm_few_prepare) : set_up(t, GEMM_TC, gemm_tc_prepare);
    if (s == FE_OK) FE_TRY(few ? launch_gemm_few(g, t->num_sms, st) : launch_gemm_tc(g, t->num_sms, st));
    return s;
}

fe_status project(const fe_target* t, const fe_project_args* a, Workspace& w, bool count, cudaStream_t st) {
    if (a->M == 0) return FE_OK;
    const int es = elem(t);
    GemmArgs g{};
    g.M = a->M;
    g.N = a->N;
    g.K = a->K;
    g.segs = 1;
    g.a[0] = a->x;
    g.b[0] = a->w;
    g.e.act = a->act;
    g.e.bias = a->bias;
    g.e.res = a->residual.p;
    g.e.res_row = a->residual.row;
    g.e.out = a->out.p;
    g.e.out_row = a->out.row;
    g.e.pre = (float*)a->pre.p;
    g.e.pre_row = a->pre.row;
    g.e.vec = (!a->bias || on16(a->bias)) && on16(a->residual, es) && on16(a->out, es) && on16(a->pre, 4);
    return gemm(t, g, w, count, st);
}

fe_status zero_rows(const fe_mat& m, int64_t rows, int64_t cols, int es, cudaStream_t st) {
    if (m.p) FE_TRY(cudaMemset2DAsync(m.p, (rows > 1 ? m.row : cols) * es, 0, cols * es, rows, st));
    return FE_OK;
}

// The products of dz (two of them: gated) that give dx and the weights' gradients.
fe_status product_gradients(const fe_target* t, int64_t M, int N, int K, const fe_mat& x, const fe_mat* w, const fe_mat* dz,
                            int n, const fe_mat& dx, const fe_mat* dw, Workspace& ws, bool count, cudaStream_t st) {
    const int es = elem(t);
    if (dx.p) {
        GemmArgs g{};
        g.M = M;
        g.N = K;
        g.K = N;
        g.segs = n;
        for (int i = 0; i < n; ++i) {
            g.a[i] = dz[i];
            g.b[i] = w[i];
        }
        g.b_t = 1;
        g.e.out = dx.p;
        g.e.out_row = dx.row;
        g.e.vec = on16(dx, es);
        const fe_status s = gemm(t, g, ws, count, st);
        if (s != FE_OK) return s;
    }
    if (dw[0].p) {
        GemmArgs g{};
        g.M = N;
        g.N = K;
        g.K = (int)M;
        g.segs = 1;
        g.twice = n == 2;
        for (int i = 0; i < n; ++i) g.a[i] = dz[i];
        g.b[0] = x;
        g.a_t = g.b_t = 1;
        g.e.out = dw[0].p;
        g.e.out_row = dw[0].row;
        g.e.vec = on16(dw[0], es) && (n == 1 || on16(dw[1], es));
        if (n == 2) {
            g.e.out2 = dw[1].p;
            g.e.out2_row = dw[1].row;
        }
        return gemm(t, g, ws, count, st);
    }
    return FE_OK;
}

fe_status project_backward(const fe_target* t, const fe_project_backward_args* a, Workspace& w, bool count, cudaStream_t st) {
    const int es = elem(t);
    if (a->M == 0) {
        if (count) return FE_OK;
        const fe_status s = zero_rows(a->dw, a->N, a->K, es, st);
        if (s != FE_OK || !a->dbias) return s;
        return zero_rows(fe_mat{a->dbias, a->N}, 1, a->N, es, st);
    }
    fe_mat dz = a->dout;
    const bool products = a->dx.p || a->dw.p, make = a->act != FE_ACT_NONE && products;
    if (make) dz = take_rows(w, a->M, a->N, es);
    if (make || a->dbias) {
        ActGradArgs g{};
        g.M = a->M;
        g.N = a->N;
        g.act = a->act;
        g.dout = a->dout;
        if (a->act != FE_ACT_NONE) g.pre = a->pre;
        if (make) g.d1 = dz;
        act_grad_plan(g, t->cfg.dtype, t->num_sms);
        if (a->dbias) g.part = (float*)w.take((int64_t)g.parts * a->N * sizeof(float));
        g.vec = on16(g.dout, es) && on16(g.pre, 4);
        if (!count) {
            FE_TRY(launch_act_grad(g, t->cfg.dtype, st));
            SumJobs sums{};
            sums.n = a->N;
            if (a->dbias) sums.add(g.part, g.parts, 1, a->dbias, a->N);
            FE_TRY(launch_sum_parts(sums, t->cfg.dtype, st));
        }
    }
    return product_gradients(t, a->M, a->N, a->K, a->x, &a->w, &dz, 1, a->dx, &a->dw, w, count, st);
}

fe_status gated(const fe_target* t, const fe_gated_ffn_args* a, Workspace& w, bool count, cudaStream_t st) {
    if (a->M == 0) return FE_OK;
    const int es = elem(t);
    GemmArgs g{};
    g.M = a->M;
    g.N = a->F;
    g.K = a->K;
    g.segs = 1;
    g.e.kind = FINISH_GATED;
    g.a[0] = a->x;
    g.b[0] = a->w_gate;
    g.b[1] = a->w_up;
    g.e.act = a->act;
    g.e.out = a->out.p;
    g.e.out_row = a->out.row;
    g.e.pre = (float*)a->gate_pre.p;
    g.e.pre_row = a->gate_pre.row;
    g.e.pre2 = (float*)a->up_pre.p;
    g.e.pre2_row = a->up_pre.row;
    g.e.vec = on16(a->out, es) && on16(a->gate_pre, 4) && on16(a->up_pre, 4);
    return gemm(t, g, w, count, st);
}

fe_status gated_backward(const fe_target* t, const fe_gated_ffn_backward_args* a, Workspace& w, bool count, cudaStream_t st) {
    const int es = elem(t);
    const fe_mat dw[2] = {a->dw_gate, a->dw_up}, weights[2] = {a->w_gate, a->w_up};
    if (a->M == 0) {
        if (count) return FE_OK;
        for (int i = 0; i < 2; ++i) {
            const fe_status s = zero_rows(dw[i], a->F, a->K, es, st);
            if (s != FE_OK) return s;
        }
        return zero_rows(a->dw_down, a->N, a->F, es, st);
    }
    const fe_mat dz[2] = {take_rows(w, a->M, a->F, es), take_rows(w, a->M, a->F, es)};
    if (a->w_down.p) {  // dh = dout w_down is finished before it is rounded
        const fe_mat h = take_rows(w, a->M, a->F, es);
        GemmArgs g{};
        g.M = a->M;
        g.N = a->F;
        g.K = a->N;
        g.segs = 1;
        g.a[0] = a->dout;
        g.b[0] = a->w_down;
        g.b_t = 1;
        g.e.kind = FINISH_GATED_GRAD;
        g.e.act = a->act;
        g.e.pre = (float*)a->gate_pre.p;
        g.e.pre_row = a->gate_pre.row;
        g.e.pre2 = (float*)a->up_pre.p;
        g.e.pre2_row = a->up_pre.row;
        g.e.out = dz[0].p;
        g.e.out2 = dz[1].p;
        g.e.out3 = h.p;
        g.e.out_row = g.e.out2_row = g.e.out3_row = h.row;
        g.e.vec = on16(a->gate_pre, 4) && on16(a->up_pre, 4);
        fe_status s = gemm(t, g, w, count, st);
        if (s != FE_OK) return s;
        const fe_mat none{};
        s = product_gradients(t, a->M, a->N, a->F, h, &a->w_down, &a->dout, 1, none, &a->dw_down, w, count, st);
        if (s != FE_OK) return s;
    } else {
        ActGradArgs g{};
        g.M = a->M;
        g.N = a->F;
        g.act = a->act;
        g.gated = 1;
        g.dout = a->dout;
        g.pre = a->gate_pre;
        g.pre2 = a->up_pre;
        g.d1 = dz[0];
        g.d2 = dz[1];
        act_grad_plan(g, t->cfg.dtype, t->num_sms);
        g.vec = on16(g.dout, es) && on16(g.pre, 4) && on16(g.pre2, 4);
        if (!count) FE_TRY(launch_act_grad(g, t->cfg.dtype, st));
    }
    return product_gradients(t, a->M, a->F, a->K, a->x, weights, dz, 2, a->dx, dw, w, count, st);
}

// Groups of rows that share gates (gate_rows may be any positive number).
int64_t gate_groups(int64_t R, int64_t gate_rows) { return R ? (R - 1) / gate_rows + 1 : 0; }

template <typename A>
bool norm_sizes_ok(const fe_target* t, const A* a) {
    if (!t || !a || a->R < 0 || a->R > kMaxRows || a->d < 1 || a->d > kMaxNorm) return false;
    if (!isfinite(a->scale) || !isfinite(a->offset) || !isfinite(a->eps) || a->eps < 0.f) return false;
    const int es = elem(t);
    if (!in_ok(a->x, es) || !opt_in(a->z, es) || !opt_in(a->gate, es) || !opt_ptr(a->post_w, es) || !opt_ptr(a->pre_w, es)) return false;
    if (!a->z.p && (a->post || a->gate.p)) return false;
    return !a->gate.p || a->gate_rows >= 1;
}

bool norm_ok(const fe_target* t, const fe_block_norm_args* a) {
    if (!norm_sizes_ok(t, a)) return false;
    const int es = elem(t);
    return (a->y.p || a->n.p) && opt_out(a->y, a->R, a->d, es) && opt_out(a->n, a->R, a->d, es);
}

bool norm_backward_ok(const fe_target* t, const fe_block_norm_backward_args* a) {
    if (!norm_sizes_ok(t, a) || (!a->dy.p && !a->dn.p)) return false;
    const int es = elem(t);
    if ((!a->z.p && a->dz.p) || (!a->gate.p && a->dgate.p) || (!a->post && a->dpost_w)) return false;
    if (!a->dx.p && !a->dz.p && !a->dgate.p && !a->dpost_w && !a->dpre_w) return false;
    const int64_t groups = a->gate.p ? gate_groups(a->R, a->gate_rows) : 0;
    return opt_in(a->dy, es) && opt_in(a->dn, es) && opt_out(a->dx, a->R, a->d, es) && opt_out(a->dz, a->R, a->d, es) &&
           opt_out(a->dgate, groups, a->d, es) && opt_ptr(a->dpost_w, es) && opt_ptr(a->dpre_w, es);
}

template <typename A>
NormArgs norm_args(const A* a) {
    NormArgs n{};
    n.R = a->R;
    n.d = a->d;
    n.post = a->post != 0;
    n.x = a->x;
    n.z = a->z;
    n.gate = a->gate;
    n.gate_rows = a->gate.p && a->gate_rows < a->R ? a->gate_rows : a->R;  // (what follows counts with sums of it and R)
    n.post_w = a->post ? a->post_w : nullptr;
    n.pre_w = a->pre_w;
    n.scale = a->scale;
    n.offset = a->offset;
    n.eps = a->eps;
    return n;
}

fe_status norm_backward(const fe_target* t, const fe_block_norm_backward_args* a, Workspace& w, bool count, cudaStream_t st) {
    const int es = elem(t);
    const fe_dtype dt = t->cfg.dtype;
    if (a->R == 0) {
        if (count) return FE_OK;
        if (a->dpost_w) FE_TRY(cudaMemsetAsync(a->dpost_w, 0, (int64_t)a->d * es, st));
        if (a->dpre_w) FE_TRY(cudaMemsetAsync(a->dpre_w, 0, (int64_t)a->d * es, st));
        return FE_OK;
    }
    NormArgs n = norm_args(a);
    n.dy = a->dy;
    n.dn = a->dn;
    n.dx = a->dx;
    n.dz = a->dz;
    n.dgate = a->dgate;
    n.vec = on16(n.x, es) && on16(n.z, es) && on16(n.gate, es) && on16(n.post_w) && on16(n.pre_w) && on16(n.dy, es) &&
            on16(n.dn, es) && on16(n.dx, es) && on16(n.dz, es) && on16(n.dgate, es);
    // (where there is no GPU the work can be counted all the same)
    const fe_status s = set_up(t, NORM_BACKWARD, [&] { return norm_backward_prepare(dt); });
    if (s != FE_OK && !count) return s;
    const int64_t workers = norm_backward_plan(n, dt, t->num_sms), bytes = workers * a->d * (int64_t)sizeof(float);
    if (a->dpre_w) n.part_pre = (float*)w.take(bytes);
    if (a->dpost_w) n.part_post = (float*)w.take(bytes);
    if (a->dgate.p && n.gate_part) n.part_gate = (float*)w.take(bytes);
    if (count) return FE_OK;
    FE_TRY(launch_block_norm_backward(n, dt, st));
    SumJobs sums{};
    sums.n = a->d;
    if (a->dpre_w) sums.add(n.part_pre, workers, 1, a->dpre_w, a->d);
    if (a->dpost_w) sums.add(n.part_post, workers, 1, a->dpost_w, a->d);
    if (a->dgate.p && n.parts) sums.add(n.part_gate, n.parts, n.groups, a->dgate.p, a->dgate.row);
    FE_TRY(launch_sum_parts(sums, dt, st));
    return FE_OK;
}

template <typename A>
bool logprob_sizes_ok(const fe_target* t, const A* a) {
    if (!t || !a || a->R < 0 || a->R > kMaxRows || a->V < 1 || a->V > kMaxRows) return false;
    if (a->J < 0 || a->J > 64 || a->K < 0 || a->K > 32 || a->K > a->V) return false;
    if (a->dtype != FE_F32 && a->dtype != FE_BF16) return false;
    if (!(a->temperature >= 0x1p-64f && a->temperature <= 0x1p64f)) return false;
    return in_ok(a->logits, a->dtype == FE_F32 ? 4 : 2);
}

template <typename A>
LogprobArgs logprob_args(const fe_target* t, const A* a) {
    LogprobArgs r{};
    r.R = a->R;
    r.V = a->V;
    r.J = a->J;
    r.K = a->K;
    r.logits = a->logits;
    r.temperature = a->temperature;
    r.tokens = a->tokens;
    r.status = t->status;
    return r;
}

// the bytes of a call's workspace, by the function that hands it out
template <typename A>
int64_t count_work(const fe_target* t, const A* a, bool ok, fe_status (*call)(const fe_target*, const A*, Workspace&, bool, cudaStream_t)) {
    if (!ok) return FE_ERR_INVALID_ARG;
    Workspace w{nullptr};
    const fe_status s = call(t, a, w, true, nullptr);
    return s != FE_OK ? s : w.used;
}

template <typename A>
fe_status run(fe_target* t, const A* a, bool ok, void* stream, fe_status (*call)(const fe_target*, const A*, Workspace&, bool, cudaStream_t)) {
    if (!ok) return FE_ERR_INVALID_ARG;
    const fe_status dv = check_device(t);
    if (dv != FE_OK) return dv;
    Workspace need{nullptr};
    fe_status s = call(t, a, need, true, nullptr);
    if (s != FE_OK) return s;
    if (!need.fits(a->work, a->work_bytes)) return FE_ERR_INVALID_ARG;
    Workspace w{(char*)a->work};
    return call(t, a, w, false, (cudaStream_t)stream);
}

}  // namespace

extern "C" {

int64_t fe_project_work(const fe_target* t, const fe_project_args* a) { return count_work(t, a, project_ok(t, a), project); }
fe_status fe_project(fe_target* t, const fe_project_args* a, void* stream) { return run(t, a, project_ok(t, a), stream, project); }

int64_t fe_project_backward_work(const fe_target* t, const fe_project_backward_args* a) {
    return count_work(t, a, project_backward_ok(t, a), project_backward);
}
fe_status fe_project_backward(fe_target* t, const fe_project_backward_args* a, void* stream) {
    return run(t, a, project_backward_ok(t, a), stream, project_backward);
}

int64_t fe_gated_ffn_work(const fe_target* t, const fe_gated_ffn_args* a) { return count_work(t, a, gated_ok(t, a), gated); }
fe_status fe_gated_ffn(fe_target* t, const fe_gated_ffn_args* a, void* stream) { return run(t, a, gated_ok(t, a), stream, gated); }

int64_t fe_gated_ffn_backward_work(const fe_target* t, const fe_gated_ffn_backward_args* a) {
    return count_work(t, a, gated_backward_ok(t, a), gated_backward);
}
fe_status fe_gated_ffn_backward(fe_target* t, const fe_gated_ffn_backward_args* a, void* stream) {
    return run(t, a, gated_backward_ok(t, a), stream, gated_backward);
}

fe_status fe_block_norm(fe_target* t, const fe_block_norm_args* a, void* stream) {
    if (!norm_ok(t, a)) return FE_ERR_INVALID_ARG;
    const fe_status dv = check_device(t);
    if (dv != FE_OK || a->R == 0) return dv;
    const int es = elem(t);
    NormArgs n = norm_args(a);
    n.y = a->y;
    n.n = a->n;
    n.vec = on16(n.x, es) && on16(n.z, es) && on16(n.gate, es) && on16(n.post_w) && on16(n.pre_w) && on16(n.y, es) && on16(n.n, es);
    const fe_status s = set_up(t, NORM, [&] { return norm_prepare(t->cfg.dtype); });
    if (s != FE_OK) return s;
    FE_TRY(launch_block_norm(n, t->cfg.dtype, t->num_sms, (cudaStream_t)stream));
    return FE_OK;
}

int64_t fe_block_norm_backward_work(const fe_target* t, const fe_block_norm_backward_args* a) {
    return count_work(t, a, norm_backward_ok(t, a), norm_backward);
}
fe_status fe_block_norm_backward(fe_target* t, const fe_block_norm_backward_args* a, void* stream) {
    return run(t, a, norm_backward_ok(t, a), stream, norm_backward);
}

fe_status fe_token_logprobs(fe_target* t, const fe_token_logprobs_args* a, void* stream) {
    if (!logprob_sizes_ok(t, a) || (a->J && (!a->tokens || !a->logprob)) || (a->K && (!a->top_id || !a->top_logprob)))
        return FE_ERR_INVALID_ARG;
    if (!a->J && !a->K && !a->entropy && !a->lse && !a->stats) return FE_ERR_INVALID_ARG;
    const fe_status dv = check_device(t);
    if (dv != FE_OK || a->R == 0) return dv;
    LogprobArgs r = logprob_args(t, a);
    r.logprob = a->logprob;
    r.entropy = a->entropy;
    r.lse = a->lse;
    r.stats = a->stats;
    r.top_id = a->top_id;
    r.top_logprob = a->top_logprob;
    const fe_status s = set_up(t, a->dtype == FE_F32 ? LOGPROBS_F32 : LOGPROBS_BF16, [&] { return logprobs_prepare(a->dtype); });
    if (s != FE_OK) return s;
    FE_TRY(launch_token_logprobs(r, a->dtype, t->num_sms, (cudaStream_t)stream));
    return FE_OK;
}

fe_status fe_token_logprobs_backward(fe_target* t, const fe_token_logprobs_backward_args* a, void* stream) {
    if (!logprob_sizes_ok(t, a) || !a->stats || !out_ok(a->dlogits, a->R, a->V, a->dtype == FE_F32 ? 4 : 2)) return FE_ERR_INVALID_ARG;
    if ((a->J && a->dlogprob && !a->tokens) || (a->K && a->dtop_logprob && !a->top_id) || (a->dentropy && !a->entropy))
        return FE_ERR_INVALID_ARG;
    const fe_status dv = check_device(t);
    if (dv != FE_OK || a->R == 0) return dv;
    LogprobArgs r = logprob_args(t, a);
    r.dlogits = a->dlogits;
    r.J = a->dlogprob ? a->J : 0;
    r.K = a->dtop_logprob ? a->K : 0;
    r.dlogprob = a->dlogprob;
    r.dentropy = a->dentropy;
    r.dlse = a->dlse;
    r.dtop = a->dtop_logprob;
    r.top_in = a->top_id;
    r.stats_in = a->stats;
    r.entropy_in = a->entropy;
    FE_TRY(launch_token_logprobs_backward(r, a->dtype, t->num_sms, (cudaStream_t)stream));
    return FE_OK;
}

}  // extern "C"
