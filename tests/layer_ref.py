"""The dense operators of a target layer in plain 64-bit form, written from their definitions
(include/fe_layer.h), their gradients by formula, and bounds of what float32 sums and the roundings of
the type may leave.

A rounding is off by at most UNIT of the value. A product of n terms summed in float32 in any order,
by adds that may truncate, is off by at most (n + 8) 2^-23 of the sum of the terms' magnitudes.
"""
import math

import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
GELU = math.sqrt(2.0 / math.pi)


def act(kind, z):
    """act(z), act'(z)."""
    if kind == "none":
        return z, torch.ones_like(z)
    if kind == "relu":
        return torch.where(z <= 0, 0.0, z), torch.where(torch.isnan(z), z, (z > 0).double())  # (NaN stays)
    if kind == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    th = torch.tanh(GELU * (z + 0.044715 * z ** 3))
    return 0.5 * z * (1 + th), 0.5 * (1 + th) + 0.5 * z * (1 - th * th) * GELU * (1 + 3 * 0.044715 * z * z)


def gamma(n):
    return (n + 8) * 2.0 ** -23


def act_slack(kind, z, dz):
    """How far act and act' are off where z is off by dz (|act'| <= 1.13, |act''| <= 1.13; relu's
    derivative jumps at 0), besides a few float32 operations."""
    if kind == "none":
        return dz, torch.zeros_like(z)
    jump = (z.abs() <= dz).double() if kind == "relu" else 1.13 * dz
    return 1.13 * dz + 2.0 ** -20 * z.abs(), jump + 2.0 ** -20 * (1 + z.abs())


class Product:
    """a [M, K] b [N, K]^T with its float32 bound."""

    def __init__(self, a, b, da=None, db=None):
        a, b = a.double(), b.double()
        self.v = a @ b.T
        self.err = gamma(a.shape[1]) * (a.abs() @ b.abs().T)
        if da is not None:
            self.err = self.err + da @ b.abs().T
        if db is not None:
            self.err = self.err + (a.abs() + (0 if da is None else da)) @ db.T


def project(c, x, w, bias, residual, dout=None):
    """c: act, unit. Returns {name: (value, bound)} of out and, with dout, dx, dw, dbias."""
    u = c["unit"]
    p = Product(x, w)
    z, dz = p.v, p.err
    if bias is not None:
        z = z + bias.double()
        dz = dz + 2.0 ** -23 * z.abs()
    a, da = act(c["act"], z)
    ea, _ = act_slack(c["act"], z, dz)
    out = a if residual is None else a + residual.double()
    got = {"out": (out, ea + 2.0 ** -23 * (a.abs() + out.abs()) + u * (out.abs() + ea))}
    if dout is not None:
        g = dout.double()
        grad = g * da
        eg = torch.zeros_like(grad)
        if c["act"] != "none":  # rounded
            _, ed = act_slack(c["act"], z, dz)
            eg = g.abs() * ed
            er = eg + u * (grad.abs() + eg)
        else:
            er = eg
        q = Product(grad, w.double().T, er)
        got["dx"] = (q.v, q.err + u * (q.v.abs() + q.err))
        q = Product(grad.T, x.double().T, er.T)
        got["dw"] = (q.v, q.err + u * (q.v.abs() + q.err))
        s, es = grad.sum(0), (gamma(grad.shape[0]) * grad.abs() + eg).sum(0)
        got["dbias"] = (s, es + u * (s.abs() + es))
    return got


def gated(c, x, wg, wu, dout=None, wd=None):
    """With wd [N, F], dout [M, N] is the gradient of the block's result behind it."""
    u = c["unit"]
    pg, pu = Product(x, wg), Product(x, wu)
    a, da = act(c["act"], pg.v)
    ea, ed = act_slack(c["act"], pg.v, pg.err)
    h = a * pu.v
    eh = ea * (pu.v.abs() + pu.err) + a.abs() * pu.err + 2.0 ** -23 * h.abs()
    eh = eh + u * (h.abs() + eh)
    got = {"out": (h, eh)}
    if dout is not None:
        g, e0 = dout.double(), 0.0
        if wd is not None:
            q = Product(g, wd.double().T)
            p = Product(g.T, h.T, db=eh.T)
            got["dw_down"] = (p.v, p.err + u * (p.v.abs() + p.err))
            g, e0 = q.v, q.err
        dg, du = g * pu.v * da, g * a
        eg = (g.abs() + e0) * ((pu.v.abs() + pu.err) * ed + pu.err * da.abs()) + e0 * (pu.v * da).abs() + 2.0 ** -22 * dg.abs()
        eu = (g.abs() + e0) * ea + e0 * a.abs() + 2.0 ** -23 * du.abs()
        eg, eu = eg + u * (dg.abs() + eg), eu + u * (du.abs() + eu)
        q = Product(torch.cat([dg, du], 1), torch.cat([wg, wu], 0).double().T, torch.cat([eg, eu], 1))
        got["dx"] = (q.v, q.err + u * (q.v.abs() + q.err))
        for name, d, e in (("dw_gate", dg, eg), ("dw_up", du, eu)):
            q = Product(d.T, x.double().T, e.T)
            got[name] = (q.v, q.err + u * (q.v.abs() + q.err))
    return got


def norm(c, x, z, post_w, gate, pre_w, dy=None, dn=None):
    """c: post, rows (a gate's), scale, offset, eps, unit. A statistic is a float32 sum, taken to be off by
    at most 2^-18 (a thread's few dozen terms and ten levels of a tree); what cancels in y counts with
    the sizes of its two parts."""
    u, R, d, o, s, t = c["unit"], x.shape[0], x.shape[1], c["offset"], c["scale"], 2.0 ** -17
    x = x.double()
    wz = 1.0 if post_w is None else post_w.double() + o
    wy = 1.0 if pre_w is None else pre_w.double() + o
    g = 1.0
    if gate is not None:
        at = torch.arange(R, device=x.device) // c["rows"]
        g = gate.double()[at]
    mean = lambda v: v.sum(1, keepdim=True) / d
    rz, zh, p = 1.0, 0.0, torch.zeros_like(x)
    if z is not None:
        z = z.double()
        p = z
        if c["post"]:
            rz = 1 / torch.sqrt(mean(z * z) + c["eps"])
            zh = z * rz
            p = zh * wz
    y = x + s * g * p
    size = x.abs() + (s * g * p).abs()
    ey = t * size
    ry = 1 / torch.sqrt(mean(y * y) + c["eps"])
    worse = 1 + torch.sqrt(mean(size * size)) * ry  # >= 1: y's parts against y
    yh = y * ry
    n = yh * wy
    en = worse * t * (n.abs() + ry * size * abs(wy)) if isinstance(wy, float) else worse * t * (n.abs() + ry * size * wy.abs())
    got = {"y": (y, ey + u * (y.abs() + ey)), "n": (n, en + u * (n.abs() + en))}
    if dy is None and dn is None:
        return got
    dx, mx = torch.zeros_like(x), torch.zeros_like(x)
    if dy is not None:
        dx, mx = dx + dy.double(), mx + dy.double().abs()
    if dn is not None:
        a = dn.double() * wy
        dx = dx + ry * (a - yh * mean(a * yh))
        mx = mx + ry * (a.abs() + ry * size * mean(a.abs() * ry * size))
        pre = dn.double() * yh
        got["dpre"] = sums(pre, dn.double().abs() * ry * size * worse * t, u)
    ex = worse * worse * t * mx
    got["dx"] = (dx, ex + u * (dx.abs() + ex))
    if z is None:
        return got
    dp, ep = s * g * dx, abs(s) * (g if isinstance(g, float) else g.abs()) * (ex + t * dx.abs())
    if gate is not None:
        parts = s * p * dx
        ge = abs(s) * p.abs() * (ex + t * dx.abs())
        groups = gate.shape[0]
        v, e, m = (torch.zeros(groups, d, dtype=torch.float64, device=x.device).index_add_(0, at, q) for q in (parts, ge, parts.abs()))
        e = e + gamma(c["rows"]) * m
        got["dgate"] = (v, e + u * (v.abs() + e))
    dz, ez = dp, ep
    if c["post"]:
        b, eb = dp * wz, ep * abs(wz) if isinstance(wz, float) else ep * wz.abs()
        dz = rz * (b - zh * mean(b * zh))
        ez = rz * (eb + t * b.abs() + zh.abs() * mean((eb + t * b.abs()) * zh.abs()))
        got["dpost"] = sums(dp * zh, ep * zh.abs() + t * (dp * zh).abs(), u)
    got["dz"] = (dz, ez + u * (dz.abs() + ez))
    return got


def sums(v, e, u):
    """Sums over the rows of v, each off by e."""
    s = v.sum(0)
    es = e.sum(0) + gamma(v.shape[0]) * v.abs().sum(0)
    return s, es + u * (s.abs() + es)


def logprobs(logits, tokens, T, top, dlogprob=None, dentropy=None, dlse=None, dtop=None, unit=2.0 ** -24, grad=False):
    """Rows [R, V], tokens [R, J]. Exponentials are off by 2^-20 and by their argument's roundings, a row's
    sum by 2^-18 (a thread's terms and a tree)."""
    x = logits.double() / T
    R, V = x.shape
    m = x.amax(1, keepdim=True)
    none = m == -math.inf
    bad = torch.isnan(x).any(1, keepdim=True) | (m == math.inf)
    base = torch.where(none, 0.0, m)
    e = torch.exp(x - base)
    z = e.sum(1, keepdim=True)
    lse = base + torch.log(z)
    fit = lambda v: torch.where(v.abs() > 3.4028235677973366e38, v.sign() * math.inf, v)  # float32's range
    lse = fit(lse)
    lse = torch.where(bad, math.nan, torch.where(none, -math.inf, lse))
    logp = torch.where(bad, math.nan, torch.where(none, -math.inf, (x - base) - torch.log(z)))
    p = torch.where(none, 0.0, e / z)
    plogp = torch.where(p > 0, p * logp, p * 0)
    H = -plogp.sum(1, keepdim=True)
    H = torch.where(none, 0.0, H)
    big = torch.where(torch.isfinite(base), base, 0.0).abs()
    elog = 2.0 ** -18 + 2.0 ** -22 * big  # of lse
    fin = lambda v: torch.where(torch.isfinite(v), v, 0.0)
    real = (tokens >= 0) & (tokens < V)
    at = tokens.long().clamp(0, V - 1)
    got = {"logprob": (torch.where(real, fit(logp.gather(1, at)), 0.0), elog + 2.0 ** -22 * fin(logp.gather(1, at)).abs()),
           "entropy": (H[:, 0], (2.0 ** -17 * (1 + fin(H).abs() + math.log(V)))[:, 0]),
           "lse": (lse[:, 0], elog[:, 0])}
    if top:
        order = torch.argsort(torch.where(torch.isnan(logits.double()), math.inf, logits.double() + 0.0), dim=1, descending=True, stable=True)
        nan_first = torch.argsort(torch.isnan(logits).gather(1, order).int(), dim=1, descending=True, stable=True)
        ids = order.gather(1, nan_first)[:, :top]
        got["top_id"] = ids.to(torch.int32)
        got["top_logprob"] = (fit(logp.gather(1, ids)), elog + 2.0 ** -22 * fin(logp.gather(1, ids)).abs())
    if grad:
        zero = lambda g, shape: torch.zeros(shape, dtype=torch.float64, device=x.device) if g is None else g.double()
        dl, dh, dz = zero(dlogprob, tokens.shape), zero(dentropy, (R,))[:, None], zero(dlse, (R,))[:, None]
        dl = torch.where(real, dl, 0.0)
        coef, sizes = torch.zeros_like(x), torch.zeros_like(x)
        coef.scatter_add_(1, at, dl)
        sizes.scatter_add_(1, at, dl.abs())
        total = dl.sum(1, keepdim=True)
        mass = dl.abs().sum(1, keepdim=True)
        if dtop is not None:
            coef.scatter_add_(1, ids, dtop.double())
            sizes.scatter_add_(1, ids, dtop.double().abs())
            total = total + dtop.double().sum(1, keepdim=True)
            mass = mass + dtop.double().abs().sum(1, keepdim=True)
        logq = torch.where(p > 0, logp, 0.0)
        g = (p * (dz - total - dh * (logq + H)) + coef) / T
        ep = 2.0 ** -18 + 2.0 ** -20 * big + 2.0 ** -22 * fin(logq).abs()
        eg = (ep * p * (dz.abs() + mass + dh.abs() * (logq.abs() + H.abs() + 1)) * 2 + 2.0 ** -20 * sizes) / T
        got["dlogits"] = (g, eg + unit * (g.abs() + eg))
    return got


def check(got, want, what=""):
    """got is within want's bound of its value, and finite, NaN or infinite where the value is."""
    v, e = want
    assert got.shape == v.shape, (what, got.shape, v.shape)
    g = got.double()
    special = ~torch.isfinite(v)
    if special.any():
        assert torch.equal(torch.isnan(g[special]), torch.isnan(v[special])), what
        inf = torch.isinf(v)
        assert torch.equal(g[inf], v[inf]), what
    far = torch.where(special, 0.0, (g - torch.where(special, 0.0, v)).abs())
    over = ~(far <= torch.where(special, 0.0, torch.as_tensor(e, dtype=torch.float64, device=g.device).expand_as(v))) & ~special
    assert not over.any(), f"{what}: {int(over.sum())} of {over.numel()} out of bounds, worst {float(torch.where(over, far, 0.0).max())}"
