"""Measured cases of the dense part of a target layer and of its answer: matrix products with bias,
activation and residual, the gated feed-forward block, the norms around a block, and the log
probabilities of given tokens, each with its backward pass.

Each case names one operator with its sizes. ``prepare`` makes the inputs on the GPU from a
seed, ``run`` is one pass through the operator (forward, or forward and backward where the case
trains): its plain form in elementary torch operations (32-bit), or, with ``own`` set, the
framework's calls. ``exact`` gives the same outputs from the definition in 64 bits.

The definitions (x, w, ... in the case's type, every sum in 32 bits or more):

  project   act(x w^T + bias) + residual
  gated     act(x w_gate^T) * (x w_up^T); with "down" also: that times w_down^T, plus residual
  norm      y = x + scale * gate * norm(z; post_weight), n = norm(y; pre_weight), where
            norm(v; w) = v / sqrt(mean(v^2) + eps) * (w + offset)
  logprobs  log softmax(logits / temperature) at the given tokens, the distribution's entropy and
            normaliser, and the most probable tokens
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def listed():
    return [
        # one token's fused query, key and value projection: plain decoding, where latency counts
        _project("project_token", M=1, K=4096, N=6144),
        # the head's logits for one draft tree
        _project("project_head", M=49, K=4096, N=128256),
        # an ordinary layer's training step: bias, activation and residual, an odd number of tokens
        _project("project_train", M=4093, K=5120, N=5120, act="gelu", bias=True, residual=True, train=True),
        # a small 32-bit model's training step (its feed-forward's way back), odd sizes
        _project("project_train_f32", M=331, K=688, N=257, dtype="f32", act="silu", bias=True, residual=True, train=True),
        # one token through a feed-forward's gate
        _gated("gated_token", M=1, K=4096, F=14336),
        # the nodes of one draft tree through a deep target's feed-forward
        _gated("gated_nodes", M=71, K=8192, F=28672),
        # a training step of the whole block: gate, up and down projection and the residual
        _gated("gated_train", M=4093, K=4096, F=14336, down=True, residual=True, train=True),
        # one token between two blocks
        _norm("norm_token", R=1, d=8192),
        # a training step's rows between two blocks, with a gate for each channel
        _norm("norm_train", R=16379, d=5120, gate="all", scale=0.5, train=True),
        # one decoded token: its log probability and the eight most probable ones
        _logprobs("logprobs_token", R=1, V=128256, top=8),
        # the nodes of 32 draft trees: the children of every node are looked up, some tokens are ruled out
        _logprobs("logprobs_nodes", R=1568, V=128256, J=8, top=10, temperature=0.7, masked=True, dtype="f32"),
        # a policy's training step: log probabilities and entropy with their gradients, padded rows
        _logprobs("logprobs_train", R=8189, V=32000, pad=True, train=True),
    ]


def _project(name=None, M=1, K=64, N=64, dtype="bf16", act="none", bias=False, residual=False, train=False):
    return _case("project", name, dict(M=M, K=K, N=N, dtype=dtype, act=act, bias=bias, residual=residual, train=train))


def _gated(name=None, M=1, K=64, F=64, dtype="bf16", act="silu", down=False, residual=False, train=False):
    return _case("gated", name, dict(M=M, K=K, F=F, dtype=dtype, act=act, down=down, residual=residual, train=train))


def _norm(name=None, R=1, d=64, dtype="bf16", gate="none", post=True, scale=1.0, offset=0.0, train=False):
    return _case("norm", name, dict(R=R, d=d, dtype=dtype, gate=gate, post=post, scale=scale, offset=offset, train=train))


def _logprobs(name=None, R=1, V=64, J=1, top=0, dtype="bf16", temperature=1.0, masked=False, pad=False, train=False):
    return _case("logprobs", name, dict(R=R, V=V, J=J, top=top, dtype=dtype, temperature=temperature, masked=masked,
                                        pad=pad, train=train))


def _case(op, name, c):
    c["op"] = op
    if name is not None:
        c["name"] = name
    return c


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A row length: most are multiples of 64 or of 8, some are odd."""
    n = _log(rng, lo, hi)
    step = rng.choice([64, 64, 8, 1])
    return max(step, n // step * step) if step > 1 else n | 1


def draw(rng):
    op = rng.choice(["project", "project", "gated", "gated", "norm", "logprobs"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    train = rng.random() < 0.5
    most = 4e12 if dtype == "bf16" else 1e11  # operations
    if op in ("project", "gated"):
        K, N = _width(rng, 64, 14336), _width(rng, 64, 14336)
        if (K % 8 or N % 8) and train:
            most = min(most, 4e11)
        per = 2.0 * K * N * (3 if train else 1) * (1 if op == "project" else 3)
        M = _log(rng, 1, max(2, min(8192, int(most / per))))
        act, residual = rng.choice(["none", "relu", "silu", "gelu"]), rng.random() < 0.5
        if op == "project":
            return _project(None, M, K, N, dtype, act, rng.random() < 0.5, residual, train)
        down = rng.random() < 0.5
        return _gated(None, M, K, N, dtype, rng.choice(["silu", "gelu", "relu"]), down, down and residual, train)
    if op == "norm":
        d = _width(rng, 64, 16384)
        return _norm(None, _log(rng, 1, max(2, int(6e7 / d))), d, dtype, rng.choice(["none", "all", "some", "each"]),
                     rng.random() < 0.75, rng.choice([1.0, 0.5, 2.5]), rng.choice([0.0, 1.0]), train)
    V = _width(rng, 64, 200000)
    return _logprobs(None, _log(rng, 1, max(2, int(1.5e8 / V))), V, rng.choice([1, 1, 3, 8]), rng.choice([0, 1, 8, 20]), dtype,
                     rng.choice([1.0, 0.7, 1.5]), rng.random() < 0.4, rng.random() < 0.4, train)


# ---- inputs -------------------------------------------------------------------------------


def _gate_rows(c):
    """Rows that share a row of gates."""
    return {"none": 0, "all": c["R"], "some": max(1, c["R"] // 5), "each": 1}[c["gate"]]


def _inputs(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = TYPES[c["dtype"]]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device=DEV) * std).to(dt)

    s = dict(case=c)
    if c["op"] == "project":
        M, K, N = c["M"], c["K"], c["N"]
        s["x"], s["w"] = normal(M, K), normal(N, K, std=K ** -0.5)
        s["bias"] = normal(N, std=0.5) if c["bias"] else None
        s["residual"] = normal(M, N) if c["residual"] else None
        s["dout"] = normal(M, N) if c["train"] else None
    elif c["op"] == "gated":
        M, K, F = c["M"], c["K"], c["F"]
        s["x"] = normal(M, K)
        s["w_gate"], s["w_up"] = normal(F, K, std=K ** -0.5), normal(F, K, std=K ** -0.5)
        s["w_down"] = normal(K, F, std=F ** -0.5) if c["down"] else None
        s["residual"] = normal(M, K) if c["residual"] else None
        s["dout"] = normal(M, K if c["down"] else F) if c["train"] else None
    elif c["op"] == "norm":
        R, d = c["R"], c["d"]
        size = torch.exp(torch.randn(R, 1, generator=g, device=DEV))  # tokens differ in magnitude
        s["x"] = (torch.randn(R, d, generator=g, device=DEV) * size).to(dt)
        s["z"] = (torch.randn(R, d, generator=g, device=DEV) * 0.3 * size.flip(0)).to(dt)
        around = 1.0 - c["offset"]
        s["post_weight"] = ((normal(d, std=0.1).float() + around).to(dt)) if c["post"] else None
        s["pre_weight"] = (normal(d, std=0.1).float() + around).to(dt)
        s["gate"] = normal(-(-R // _gate_rows(c)), d, std=0.5) if c["gate"] != "none" else None
        s["dy"], s["dn"] = (normal(R, d), normal(R, d)) if c["train"] else (None, None)
    else:
        R, V, J = c["R"], c["V"], c["J"]
        x = torch.randn(R, V, generator=g, device=DEV) * 2.5
        if c["masked"]:
            x.masked_fill_(torch.rand(R, V, generator=g, device=DEV) < 0.3, -math.inf)
        x[:, 0] = 1.0  # (every row keeps a token)
        s["logits"] = x.to(dt)
        tokens = torch.randint(0, V, (R, J), generator=g, device=DEV, dtype=torch.int32)
        tokens[:, :1] = torch.where(torch.isinf(x.gather(1, tokens[:, :1].long())), 0, tokens[:, :1])
        if c["pad"]:
            tokens[torch.rand(R, generator=g, device=DEV) < 0.2] = -1
        s["tokens"] = tokens
        if c["train"]:
            s["dlogprob"] = torch.randn(R, J, generator=g, device=DEV)
            s["dentropy"] = torch.randn(R, generator=g, device=DEV) * 0.1
    return s


# the inputs that a training step differentiates, in the order of run's gradients
_LEAVES = {"project": ("x", "w", "bias", "residual"), "gated": ("x", "w_gate", "w_up", "w_down", "residual"),
           "norm": ("x", "z", "post_weight", "gate", "pre_weight"), "logprobs": ("logits",)}


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2509_20416_gb300 as fe
        s["fe"] = fe
        s["target"] = fe.fe_target_init(dict(n_heads=1, n_kv_heads=1, head_dim=64, max_seq=16, dtype=case["dtype"],
                                             rope_theta=1e4))
        s["leaves"] = [s[k] for k in _LEAVES[case["op"]] if s.get(k) is not None]
        if case["train"]:
            for x in s["leaves"]:
                x.requires_grad_()
    return s


# ---- the plain forms ----------------------------------------------------------------------


def _act(kind, z):
    """An activation and its derivative (gelu: the tanh form)."""
    if kind == "none":
        return z, torch.ones_like(z)
    if kind == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    if kind == "silu":
        p = 1 / (1 + torch.exp(-z))
        return z * p, p * (1 + z * (1 - p))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z * z * z))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)


def _plain_project(s):
    c = s["case"]
    x, w, dt = s["x"].float(), s["w"].float(), s["x"].dtype
    z = x @ w.T
    if s["bias"] is not None:
        z = z + s["bias"].float()
    a, da = _act(c["act"], z)
    y = a if s["residual"] is None else a + s["residual"].float()
    out = [y.to(dt)]
    if c["train"]:
        dz = s["dout"].float() * da
        out += [(dz @ w).to(dt), (dz.T @ x).to(dt)]
        if s["bias"] is not None:
            out.append(dz.sum(0).to(dt))
        if s["residual"] is not None:
            out.append(s["dout"])
    return out


def _plain_gated(s):
    c = s["case"]
    x, wg, wu, dt = s["x"].float(), s["w_gate"].float(), s["w_up"].float(), s["x"].dtype
    zg, zu = x @ wg.T, x @ wu.T
    a, da = _act(c["act"], zg)
    h = a * zu
    y = h
    if c["down"]:
        wd = s["w_down"].float()
        y = h @ wd.T
        if s["residual"] is not None:
            y = y + s["residual"].float()
    out = [y.to(dt)]
    if c["train"]:
        dy = s["dout"].float()
        dh = dy @ wd if c["down"] else dy
        dg, du = dh * zu * da, dh * a
        out += [(dg @ wg + du @ wu).to(dt), (dg.T @ x).to(dt), (du.T @ x).to(dt)]
        if c["down"]:
            out.append((dy.T @ h).to(dt))
        if s["residual"] is not None:
            out.append(s["dout"])
    return out


def _plain_norm(s):
    c = s["case"]
    dt, d, R, o, k = s["x"].dtype, c["d"], c["R"], c["offset"], c["scale"]
    x, z = s["x"].float(), s["z"].float()
    per = _gate_rows(c)
    at = torch.arange(R, device=DEV) // max(per, 1)
    g = s["gate"].float()[at] if per else 1.0
    if c["post"]:
        wz = s["post_weight"].float() + o
        rz = 1 / torch.sqrt((z * z).sum(1, keepdim=True) / d + EPS)
        zh = z * rz
        p = zh * wz
    else:
        p = z
    y = x + k * g * p
    wy = s["pre_weight"].float() + o
    ry = 1 / torch.sqrt((y * y).sum(1, keepdim=True) / d + EPS)
    yh = y * ry
    out = [y.to(dt), (yh * wy).to(dt)]
    if c["train"]:
        dn = s["dn"].float()
        dyh = dn * wy
        dx = s["dy"].float() + ry * (dyh - yh * (dyh * yh).sum(1, keepdim=True) / d)
        dp = k * g * dx
        dz = dp
        if c["post"]:
            dzh = dp * wz
            dz = rz * (dzh - zh * (dzh * zh).sum(1, keepdim=True) / d)
        out += [dx.to(dt), dz.to(dt)]
        if c["post"]:
            out.append((dp * zh).sum(0).to(dt))
        if per:
            dg = torch.zeros(s["gate"].shape, device=DEV).index_add_(0, at, k * p * dx) if per > 1 else k * p * dx
            out.append(dg.to(dt))
        out.append((dn * yh).sum(0).to(dt))
    return out


def _keys(x):
    """Whole numbers that order the elements of rows as their values, the smaller index first."""
    bits = (x + 0.0).view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    return order * 2 ** 32 + (2 ** 32 - 1 - torch.arange(x.shape[1], device=x.device))


def _plain_logprobs(s):
    c = s["case"]
    x = s["logits"].float() / c["temperature"]
    tok = s["tokens"].long()
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    z = e.sum(1, keepdim=True)
    lse = m + torch.log(z)
    p = e / z
    logp = x - lse
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(1)
    real = tok >= 0
    out = [torch.where(real, logp.gather(1, tok.clamp(min=0)), 0.0), entropy, lse[:, 0]]
    if c["top"]:
        key = torch.topk(_keys(s["logits"].float()), min(c["top"], c["V"]), 1).values
        top = 2 ** 32 - 1 - (key & (2 ** 32 - 1))
        out += [top.to(torch.int32), logp.gather(1, top)]
    if c["train"]:
        d = torch.where(real, s["dlogprob"], 0.0)
        h = s["dentropy"][:, None]
        g = -p * (d.sum(1, keepdim=True) + h * (torch.where(p > 0, logp, 0.0) + entropy[:, None]))
        g.scatter_add_(1, tok.clamp(min=0), d)
        out.append((g / c["temperature"]).to(s["logits"].dtype))
    return out


def run(state):
    s = state
    c = s["case"]
    if not own:
        return {"project": _plain_project, "gated": _plain_gated, "norm": _plain_norm, "logprobs": _plain_logprobs}[c["op"]](s)
    fe, t = s["fe"], s["target"]
    if c["op"] == "project":
        out = [fe.fe_project(t, s["x"], s["w"], bias=s["bias"], act=c["act"], residual=s["residual"])]
    elif c["op"] == "gated":
        out = [fe.fe_gated_ffn(t, s["x"], s["w_gate"], s["w_up"], w_down=s["w_down"], act=c["act"], residual=s["residual"])]
    elif c["op"] == "norm":
        out = list(fe.fe_block_norm(t, s["x"], s["z"], post=c["post"], post_weight=s["post_weight"], gate=s["gate"],
                                    gate_rows=_gate_rows(c), scale=c["scale"], pre_weight=s["pre_weight"],
                                    offset=c["offset"], eps=EPS))
    else:
        out = list(fe.fe_token_logprobs(t, s["logits"], s["tokens"], top=min(c["top"], c["V"]), temperature=c["temperature"]))
        out = out if c["top"] else out[:3]
    if c["train"]:
        given = {"norm": ("dy", "dn"), "logprobs": ("dlogprob", "dentropy")}.get(c["op"], ("dout",))
        grads = torch.autograd.grad(out[:len(given)], s["leaves"], [s[k] for k in given])
        out = [x.detach() for x in out] + list(grads)
    return out


# ---- what a pass cannot do without ----------------------------------------------------------


def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    n = 3 if c["train"] else 1
    if c["op"] == "project":
        M, K, N = c["M"], c["K"], c["N"]
        rows, weights = M * N, N * K + (N if c["bias"] else 0)
        byt = M * K + weights + rows * (2 if c["residual"] else 1)
        if c["train"]:  # read dout; write the gradients of x, w, bias
            byt += rows + M * K + weights
        return {"bytes": byt * es, "flops": 2 * n * M * N * K}
    if c["op"] == "gated":
        M, K, F = c["M"], c["K"], c["F"]
        rows, weights = M * (K if c["down"] else F), (3 if c["down"] else 2) * F * K
        byt = M * K + weights + rows * (2 if c["residual"] else 1)
        if c["train"]:
            byt += rows + M * K + weights
        return {"bytes": byt * es, "flops": 2 * n * M * weights}
    if c["op"] == "norm":
        R, d = c["R"], c["d"]
        weights = d * (2 if c["post"] else 1) + (s_rows(c) * d)
        byt = 4 * R * d + weights
        if c["train"]:  # read dy, dn; write the gradients of x, z and the weights
            byt += 4 * R * d + weights
        return {"bytes": byt * es, "flops": (40 if c["train"] else 12) * R * d}
    R, V = c["R"], c["V"]
    byt = R * V * es * (2 if c["train"] else 1) + 4 * R * (2 * c["J"] + 2 + 2 * c["top"]) + (4 * R * (c["J"] + 1) if c["train"] else 0)
    return {"bytes": byt, "flops": (20 if c["train"] else 8) * R * V}


def s_rows(c):
    """Rows of gates."""
    per = _gate_rows(c)
    return -(-c["R"] // per) if per else 0


# ---- the definition in 64 bits ---------------------------------------------------------------


def _exact_act(kind, z):
    if kind == "none":
        return z
    if kind == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if kind == "silu":
        return z * torch.sigmoid(z)
    u = 2.0 * math.sqrt(2.0 / math.pi) * z * (1.0 + 0.044715 * z ** 2)
    return z * torch.sigmoid(u)  # (1 + tanh(u / 2)) / 2 = sigmoid(u)


def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    if c["op"] == "logprobs":
        return _exact_logprobs(c, s)
    if c["op"] != "norm" and work(c)["flops"] > 8e12:
        return None
    names = [k for k in _LEAVES[c["op"]] if s.get(k) is not None]
    v = {k: s[k].double().requires_grad_(c["train"]) for k in names}
    if c["op"] == "project":
        z = torch.einsum("mk,nk->mn", v["x"], v["w"])
        y = _exact_act(c["act"], z + v["bias"] if "bias" in v else z)
        outs, given = [y + v["residual"] if "residual" in v else y], ["dout"]
    elif c["op"] == "gated":
        y = _exact_act(c["act"], torch.einsum("mk,nk->mn", v["x"], v["w_gate"])) * torch.einsum("mk,nk->mn", v["x"], v["w_up"])
        y = torch.einsum("mf,kf->mk", y, v["w_down"]) if c["down"] else y
        outs, given = [y + v["residual"] if "residual" in v else y], ["dout"]
    else:
        def rms(a, w):
            return a * (a.square().mean(-1, keepdim=True) + EPS).rsqrt() * (w + c["offset"])
        b = rms(v["z"], v["post_weight"]) if c["post"] else v["z"]
        if "gate" in v:
            b = b * v["gate"].repeat_interleave(_gate_rows(c), 0)[:c["R"]]
        y = v["x"] + c["scale"] * b
        outs, given = [y, rms(y, v["pre_weight"])], ["dy", "dn"]
    out = [o.detach() for o in outs]
    if c["train"]:
        out += torch.autograd.grad(outs, [v[k] for k in names], [s[k].double() for k in given])
    return out


def _exact_logprobs(c, s):
    R, V, T, k = c["R"], c["V"], c["temperature"], min(c["top"], c["V"])
    cols = [[] for _ in range(3 + (2 if k else 0) + (1 if c["train"] else 0))]
    step = max(1, int(1e8 // V))
    for r in range(0, R, step):
        x = s["logits"][r:r + step].double()
        tok = s["tokens"][r:r + step].long()
        logp = torch.log_softmax(x / T, 1)
        p = logp.exp()
        plogp = torch.where(p > 0, p * logp, torch.zeros_like(p))
        lp = torch.zeros(tok.shape, dtype=torch.float64, device=DEV)
        for j in range(c["J"]):
            has = tok[:, j] >= 0
            lp[has, j] = logp[has, tok[has, j]]
        parts = [lp, -plogp.sum(1), torch.logsumexp(x / T, 1)]
        if k:
            i = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
            parts += [i.to(torch.int32), logp.gather(1, i)]
        if c["train"]:  # the gradient of log p, then through the softmax
            g = -s["dentropy"][r:r + step, None].double() * (plogp + p)
            for j in range(c["J"]):
                has = (tok[:, j] >= 0).nonzero()[:, 0]
                g[has, tok[has, j]] += s["dlogprob"][r + has, j].double()
            parts.append((g - p * g.sum(1, keepdim=True)) / T)
        for a, b in zip(cols, parts):
            a.append(b)
    return [torch.cat(a) for a in cols]
