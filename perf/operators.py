"""Measured cases of the target-side operators: rotary positions, the (quantised) key/value
cache's write and read, moving accepted rows, and attention of a draft tree over the cache.

Each case names one operator with its sizes. ``prepare`` makes the inputs on the GPU from a
seed, ``run`` is one pass through the operator: its plain form in elementary torch operations
(32-bit), or, with ``own`` set, the framework's calls. ``exact`` gives the same outputs from
the definition in 64 bits.

Quantised caches hold each row of a head as e4m3 numbers times the smallest power of two that
lets the row's largest magnitude fit (448 is the largest e4m3 number), so a row reads back
exactly in bfloat16.
"""
import math

import torch

own = False

DEV = "cuda"
F8 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": F8}

# the head layouts of the framework's drafter shapes: (query heads, key/value heads, head size)
HEADS = [(40, 40, 128), (32, 8, 128), (64, 8, 128), (4, 4, 64)]


def _base(op, **kw):
    c = dict(op=op, B=1, T=1, H=32, Hkv=8, hd=128, p_lo=0, p_hi=0, page=0, dtype="bf16", cache="bf16", mask="tree",
             ragged=False, rot=128, layout="half", scaling="none", theta=5e5, backward=False, layers=1)
    c.update(kw)
    return c


def listed():
    return [
        # the queries and keys of one draft tree (7 levels of 10 under the root), one user
        _base("rope", name="rope_step", T=71, H=64, p_lo=2047, p_hi=2047, scaling="bands"),
        # gradients of rotated rows over odd-length training sequences: half the head rotated,
        # interleaved pairs, a context stretched eightfold
        _base("rope", name="rope_train_f32", B=4, T=4093, H=32, dtype="f32", rot=64, layout="interleaved",
              scaling="yarn", theta=1e4, backward=True),
        # one cycle's tree rows of 32 users into an 8-bit paged cache, rotated on the way, and back
        _base("cache", name="cache_step_e4m3", B=32, T=49, p_lo=256, p_hi=4096, page=16, cache="e4m3"),
        # a prompt chunk of every head's rows into a 16-bit cache
        _base("cache", name="cache_chunk_bf16", B=2, T=1021, H=40, Hkv=40, p_lo=333, p_hi=900, theta=1e4),
        # long prompts into an 8-bit cache and back (moving a user between machines)
        _base("cache", name="cache_prompt_e4m3", B=4, T=8191, H=64, p_lo=0, p_hi=130, page=64, cache="e4m3"),
        # accepted rows of all layers of a deep target to their places, one user
        _base("keep", name="keep_b1_bf16", T=81, H=64, p_lo=257, p_hi=257, layers=80),
        # the same for 32 users with page tables
        _base("keep", name="keep_b32_bf16", B=32, T=49, p_lo=100, p_hi=700, page=16, layers=32),
        # one token of one user: plain decoding, where latency counts
        _base("attn", name="attn_token", T=1, p_lo=199, p_hi=199, mask="causal"),
        # draft trees of 32 users of mixed lengths, paged 16-bit cache
        _base("attn", name="attn_tree_b32", B=32, T=49, p_lo=256, p_hi=4096, page=16),
        # a draft tree at the end of a long document, 8-bit cache
        _base("attn", name="attn_tree_long_e4m3", T=81, H=64, p_lo=130944, p_hi=130944, cache="e4m3"),
        # a prompt chunk of a model without shared heads
        _base("attn", name="attn_chunk", B=2, T=1021, H=40, Hkv=40, p_lo=1500, p_hi=2500, mask="causal"),
        # 32-bit trees of a small model (64-wide heads), used to check a target
        _base("attn", name="attn_tree_f32", B=4, T=13, H=4, Hkv=4, hd=64, rot=64, p_lo=64, p_hi=1500, dtype="f32", cache="f32",
              ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "cache", "keep", "attn", "attn", "attn"])
    H, Hkv, hd = rng.choice(HEADS)
    c = _base(op, H=H, Hkv=Hkv, hd=hd, theta=rng.choice([1e4, 5e5]), dtype=rng.choice(["bf16", "bf16", "f32"]),
              page=rng.choice([0, 0, 16, 64, 24, 5]))
    c["rot"] = rng.choice([hd, hd, hd // 2])
    c["cache"] = c["dtype"] if c["dtype"] == "f32" else rng.choice(["bf16", "e4m3"])
    c["layout"] = rng.choice(["half", "interleaved"])
    c["scaling"] = rng.choice(["none", "linear", "ntk", "bands", "yarn"])
    if op == "rope":
        c["B"] = _log(rng, 1, 16)
        c["T"] = _log(rng, 1, max(2, 16000 // c["B"]))
        c["backward"] = rng.random() < 0.5
        c["p_hi"] = rng.choice([0, 5000])
    elif op == "cache":
        c["B"] = _log(rng, 1, 32)
        c["T"] = _log(rng, 1, max(2, 12000 // c["B"]))
        c["p_hi"] = _log(rng, 1, 4000)
        c["p_lo"] = rng.randint(0, c["p_hi"])
        c["page"] = rng.choice([0, 16, 64, 24, 5])
    elif op == "keep":
        c["dtype"] = "bf16"
        c["cache"] = "bf16"
        c["B"] = _log(rng, 1, 32)
        c["T"] = _log(rng, 2, 120)
        c["layers"] = _log(rng, 1, 40)
        c["p_hi"] = _log(rng, 1, 500)
        c["p_lo"] = rng.randint(0, c["p_hi"])
    else:
        c["B"] = _log(rng, 1, 32)
        c["T"] = _log(rng, 1, 160)
        c["p_hi"] = _log(rng, 1, (60000 if c["dtype"] == "bf16" else 8000) // c["B"] + 2)
        c["p_lo"] = rng.randint(0, c["p_hi"])
        c["mask"] = rng.choice(["tree", "causal"])
        c["ragged"] = rng.random() < 0.4
    return c


# ---- inputs -------------------------------------------------------------------------------


def _lens(c):
    """Each sequence's rows before this step: spread evenly over the case's range."""
    B = c["B"]
    return [c["p_lo"] + (c["p_hi"] - c["p_lo"]) * b // max(1, B - 1) for b in range(B)]


def _cap(c):
    return ((max(_lens(c)) + c["T"] + 15) // 16) * 16


def _quant(x):
    """float32 rows [..., hd] -> (e4m3 numbers, float32 power-of-two scale per row)."""
    m, e = torch.frexp(x.abs().amax(-1))
    k = torch.clamp(torch.where(m <= 0.875, e - 9, e - 8), -120, 120)
    s = torch.ldexp(torch.ones_like(m), k)
    return (x / s[..., None]).to(F8), s


def _freqs(c):
    """Angle per position of each rotated pair, and the amplitude (float64 on the CPU)."""
    rd, theta = c["rot"], c["theta"]
    i = torch.arange(0, rd, 2, dtype=torch.float64)
    f, amp, kind = theta ** (-i / rd), 1.0, c["scaling"]
    factor, orig = 8.0, 8192.0
    if kind == "linear":
        f = f / factor
    elif kind == "ntk":
        f = (theta * factor ** (rd / (rd - 2))) ** (-i / rd)
    elif kind == "bands":
        lo, hi = 1.0, 4.0
        smooth = torch.clamp((orig * f / (2 * math.pi) - lo) / (hi - lo), 0, 1)
        f = f * ((1 - smooth) / factor + smooth)
    elif kind == "yarn":
        def dim(turns):
            return rd * math.log(orig / (turns * 2 * math.pi)) / (2 * math.log(theta))
        lo, hi = max(math.floor(dim(32.0)), 0), min(math.ceil(dim(1.0)), rd - 1)
        ramp = torch.clamp((i / 2 - lo) / max(hi - lo, 0.001), 0, 1)
        f, amp = f * (ramp / factor + 1 - ramp), 0.1 * math.log(factor) + 1
    return f, amp


def _inputs(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt, B, T, H, Hkv, hd = TYPES[c["dtype"]], c["B"], c["T"], c["H"], c["Hkv"], c["hd"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    s = dict(case=c)
    # the step's projections lie side by side in one row, as a fused projection leaves them
    qkv = normal(B, T, (H + 2 * Hkv), hd)
    qkv[:, :, :H] *= 0.5 + 2.0 * torch.rand(H, 1, generator=g, device=DEV)
    qkv = qkv.to(dt)
    s["q"], s["k"], s["v"] = qkv[:, :, :H], qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:]
    order = torch.randperm(B, generator=g, device=DEV)
    lens = torch.tensor(_lens(c), device=DEV, dtype=torch.int32)[order].contiguous()
    s["start"] = lens
    depth = torch.arange(T, device=DEV, dtype=torch.int32)
    s["pos"] = (lens[:, None] + depth).contiguous()
    if c["op"] == "rope":
        return s
    cap, page, Ly = _cap(c), c["page"], c["layers"]
    if page:
        per = -(-cap // page)
        n = B * per + 3
        perm = torch.randperm(n, generator=g, device=DEV)[:B * per]
        s["table"], s["n_pages"] = perm.to(torch.int32).view(B, per).contiguous(), n
        shape = (n, Hkv, page, hd)
    else:
        s["table"], s["n_pages"] = None, 0
        shape = (B, Hkv, cap, hd)
    for name in ("k", "v"):
        x = torch.empty((Ly,) + shape, dtype=dt, device=DEV)
        x.normal_(generator=g)
        if c["cache"] == "e4m3":
            x, scale = _quant(x.float())
            s[name + "_scale"] = scale
        s[name + "_cache"] = x
    if c["op"] == "cache":
        s["nodes"] = torch.full((B,), T, dtype=torch.int32, device=DEV)
    if c["op"] == "attn":
        if c["mask"] == "tree":  # random trees: node i's parent is an earlier node, often a recent one
            u = torch.rand(B, T, generator=g, device=DEV)
            idx = torch.arange(T, device=DEV)
            parent = (idx * (1 - 0.5 * u * u)).long().clamp(max=T - 1)
            parent = torch.minimum(parent, (idx - 1).clamp(min=0))
            reach = torch.zeros(B, T, T, device=DEV).scatter_(2, parent.expand(B, T)[..., None], 1.0)
            reach = ((reach + torch.eye(T, device=DEV)) > 0).float()
            for _ in range(max(1, math.ceil(math.log2(T + 1)))):
                reach = ((reach @ reach) > 0).float()
            s["mask"] = reach.to(torch.uint8).contiguous()
        else:
            s["mask"] = None
        nodes = torch.full((B,), T, dtype=torch.int32, device=DEV)
        if c["ragged"]:
            nodes = torch.randint(1, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        s["nodes"] = nodes
    if c["op"] == "keep":  # accepted nodes of each tree: growing node numbers, some walks short
        n = min(T - 1, 8)
        pick = torch.rand(B, T - 1, generator=g, device=DEV).argsort(1)[:, :n].sort(1).values + 1
        s["path"] = pick.to(torch.int32).contiguous()
        s["accept"] = torch.randint(0, n + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        s["accept"][0] = n
    return s


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    if own:
        import paper_2509_20416_gb300 as fe
        s["fe"] = fe
        s["target"] = fe.fe_target_init(dict(
            n_heads=c["H"], n_kv_heads=c["Hkv"], head_dim=c["hd"], max_batch=c["B"], max_seq=_cap(c),
            page_size=c["page"], dtype=c["dtype"], cache_dtype=c["cache"] if c["op"] != "rope" else c["dtype"],
            rope_theta=c["theta"], rope_dim=c["rot"], rope_layout=c["layout"], rope_scaling=c["scaling"],
            rope_factor=8.0, rope_orig=8192.0,
            rope_low=32.0 if c["scaling"] == "yarn" else 1.0, rope_high=1.0 if c["scaling"] == "yarn" else 4.0))
        if c["op"] != "rope":
            s["cache"] = fe.Cache(s["target"], s["k_cache"], s["v_cache"], s.get("k_scale"), s.get("v_scale"),
                                  page_table=s["table"], n_pages=s["n_pages"])
    else:
        f, amp = _freqs(c)
        a = torch.arange(_cap(c), dtype=torch.float64, device=DEV)[:, None] * f.to(DEV)
        s["cos"], s["sin"] = (a.cos() * amp).float(), (a.sin() * amp).float()
    s["L"] = _cap(c)
    return s


# ---- the plain forms ----------------------------------------------------------------------


def _rotate(c, x, cos, sin):
    """x [B, T, heads, hd] in any float type with cos, sin [B, T, 1, rot / 2] of the same."""
    rd = c["rot"]
    r = x[..., :rd]
    if c["layout"] == "half":
        a, b = r[..., :rd // 2], r[..., rd // 2:]
    else:
        a, b = r[..., 0::2], r[..., 1::2]
    u, w = a * cos - b * sin, b * cos + a * sin
    y = torch.cat([u, w], -1) if c["layout"] == "half" else torch.stack([u, w], -1).flatten(-2)
    return torch.cat([y, x[..., rd:]], -1)


def _where(s, slots):
    """Index of cache rows (b, slot) for slots [B, n]: into dimensions 0 (page or sequence) and 2."""
    page = s["case"]["page"]
    if page:
        return s["table"].long().gather(1, slots // page), slots % page
    return torch.arange(slots.shape[0], device=DEV)[:, None].expand_as(slots), slots


def _get(s, name, slots, layer=0):
    """Cache rows at slots [B, n] as float32 [B, n, Hkv, hd]."""
    i, j = _where(s, slots)
    x = s[name + "_cache"][layer][i, :, j].float()
    if s["case"]["cache"] == "e4m3":
        x = x * s[name + "_scale"][layer][i, :, j][..., None]
    return x


def _put(s, name, slots, rows):
    """Write float32 rows [B, n, Hkv, hd] at slots [B, n]."""
    i, j = _where(s, slots)
    cache = s[name + "_cache"][0]
    if s["case"]["cache"] == "e4m3":
        rows, scale = _quant(rows)
        s[name + "_scale"][0][i, :, j] = scale
        cache.view(torch.uint8)[i, :, j] = rows.view(torch.uint8)
    else:
        cache[i, :, j] = rows.to(cache.dtype)


def _plain_rope(s):
    c, p = s["case"], s["pos"].long()
    cos, sin = s["cos"][p][:, :, None], s["sin"][p][:, :, None]
    sin = -sin if c["backward"] else sin
    return [_rotate(c, x.float(), cos, sin).to(x.dtype) for x in (s["q"], s["k"])]


def _plain_cache(s):
    c = s["case"]
    q, k = _rotate_qk(s)
    slots = s["start"].long()[:, None] + torch.arange(c["T"], device=DEV)
    _put(s, "k", slots, k)
    _put(s, "v", slots, s["v"].float())
    return [q.to(s["q"].dtype), _get(s, "k", slots).to(s["k"].dtype), _get(s, "v", slots).to(s["v"].dtype)]


def _rotate_qk(s):
    c, p = s["case"], s["pos"].long()
    cos, sin = s["cos"][p][:, :, None], s["sin"][p][:, :, None]
    return _rotate(c, s["q"].float(), cos, sin), _rotate(c, s["k"].float(), cos, sin)


def _plain_keep(s):
    n = s["path"].shape[1]
    j = torch.arange(n, device=DEV)
    live = (j < s["accept"][:, None])
    start = s["start"].long()[:, None]
    dst = start + 1 + j
    src = torch.where(live, start + s["path"].long(), dst)  # a row past the accepted ones stays as it is
    i0, j0 = _where(s, src)
    i1, j1 = _where(s, dst)
    s["k_cache"][:, i1, :, j1] = s["k_cache"][:, i0, :, j0]
    s["v_cache"][:, i1, :, j1] = s["v_cache"][:, i0, :, j0]
    return [s["k_cache"], s["v_cache"]]


def _plain_attn(s):
    c = s["case"]
    B, T, H, Hkv, hd, L = c["B"], c["T"], c["H"], c["Hkv"], c["hd"], s["L"]
    G = H // Hkv
    slot = torch.arange(L, device=DEV)
    P, n = s["start"].long()[:, None, None], s["nodes"].long()[:, None, None]
    node = torch.arange(T, device=DEV)[:, None]
    rel = slot - P  # [B, 1, L]: a slot's node number
    if s["mask"] is not None:
        inside = s["mask"].bool().gather(2, rel.clamp(0, T - 1).expand(B, T, L))
    else:
        inside = rel <= node
    ok = ((rel < 0) | (inside & (rel < n))) & (node < n)
    last = (P[:, :, 0] + n[:, :, 0] - 1).clamp(min=0)
    slots = torch.minimum(slot.expand(B, L), last)
    k, v = _get(s, "k", slots).permute(0, 2, 3, 1), _get(s, "v", slots).transpose(1, 2)
    q = s["q"].float().view(B, T, Hkv, G, hd).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * T, hd)
    x = (q @ k).view(B, Hkv, G, T, L) * (1.0 / math.sqrt(hd))
    x = torch.where(ok[:, None, None], x, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(x - m)
    z = p.sum(-1, keepdim=True)
    o = (p.view(B, Hkv, G * T, L) @ v).view(B, Hkv, G, T, hd) / torch.where(z == 0, 1.0, z)
    lse = (m + torch.log(z)).squeeze(-1)
    return [o.permute(0, 3, 1, 2, 4).reshape(B, T, H, hd).to(s["q"].dtype), lse.permute(0, 3, 1, 2).reshape(B, T, H)]


def run(state):
    s = state
    c = s["case"]
    op = c["op"]
    if not own:
        return {"rope": _plain_rope, "cache": _plain_cache, "keep": _plain_keep, "attn": _plain_attn}[op](s)
    fe, t = s["fe"], s["target"]
    if op == "rope":
        return list(fe.fe_rope(t, s["q"], s["k"], s["pos"], backward=c["backward"]))
    if op == "cache":
        q = fe.fe_cache_write(t, s["cache"], 0, s["k"], s["v"], s["start"], pos=s["pos"], q=s["q"])
        return [q] + list(fe.fe_cache_read(t, s["cache"], 0, s["start"], s["nodes"], c["T"]))
    if op == "keep":
        fe.fe_cache_keep(t, s["cache"], s["path"], s["accept"], s["start"])
        return [s["k_cache"], s["v_cache"]]
    return list(fe.fe_tree_attention(t, s["cache"], 0, s["q"], s["start"], mask=s["mask"], n_nodes=s["nodes"]))


# ---- what a pass cannot do without ----------------------------------------------------------


def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    B, T, H, Hkv, hd = c["B"], c["T"], c["H"], c["Hkv"], c["hd"]
    row = hd + 4 if c["cache"] == "e4m3" else hd * es  # a cached row of a head
    rows = B * T
    if c["op"] == "rope":
        return {"bytes": 2 * rows * (H + Hkv) * hd * es + 4 * rows, "flops": 3 * rows * (H + Hkv) * c["rot"]}
    if c["op"] == "cache":
        # read q, k, v; write q and the cache rows; read those and write them out
        step = rows * (2 * H + 2 * Hkv) * hd * es + 2 * rows * Hkv * row
        return {"bytes": step + rows * 2 * Hkv * (row + hd * es), "flops": 3 * rows * (H + Hkv) * c["rot"]}
    if c["op"] == "keep":
        n = min(T - 1, 8)
        moved = n + (B - 1) * n / 2  # rows of one head of one layer
        return {"bytes": c["layers"] * 2 * Hkv * moved * 2 * row, "flops": 0}
    kv = sum(_lens(c))
    seen = sum(p + (0.5 * (T + 1) if c["mask"] == "causal" else T) for p in _lens(c))
    byt = 2 * rows * H * hd * es + 4 * rows * H + (kv + rows) * 2 * Hkv * row + (B * T * T if c["mask"] == "tree" else 0)
    return {"bytes": byt, "flops": 4 * T * H * hd * seen}


# ---- the definition in 64 bits ---------------------------------------------------------------


def _exact_rot(c, x, pos):
    """Rotate pair by pair as complex numbers: x [B, T, heads, hd], pos [B, T]."""
    f, amp = _freqs(c)
    x = x.double().clone()
    ang = pos.double()[..., None] * f.to(x.device)
    turn = torch.polar(torch.full_like(ang, amp), -ang if c["backward"] else ang)[:, :, None]
    h = c["rot"] // 2
    lo = torch.arange(h, device=x.device)
    i, j = (lo, lo + h) if c["layout"] == "half" else (2 * lo, 2 * lo + 1)
    z = torch.complex(x[..., i], x[..., j]) * turn
    x[..., i], x[..., j] = z.real, z.imag
    return x


def _exact_stored(c, x):
    """What a cache of the case's type holds for float64 rows x."""
    if c["cache"] != "e4m3":
        return x.to(TYPES[c["cache"]]).double()

    def two(k):  # 2^k for whole numbers (a power in 64 bits on the GPU may be off by a rounding)
        return torch.ldexp(torch.ones(k.shape, device=k.device), k.int()).double()

    top = x.abs().amax(-1, keepdim=True)
    k = torch.ceil(torch.log2(top / 448.0).clamp(min=-120))
    k = torch.where(448.0 * two(k - 1) >= top, k - 1, k)  # (a logarithm just above a whole number)
    k = torch.where(448.0 * two(k) < top, k + 1, k).clamp(min=-120)
    y = x / two(k)
    step = two(torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent - 4)
    return torch.round(y / step) * step * two(k)


def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    if c["op"] == "rope":
        return [_exact_rot(c, s["q"], s["pos"]), _exact_rot(c, s["k"], s["pos"])]
    if c["op"] == "cache":
        if c["B"] * c["T"] * c["H"] * c["hd"] > 3e8:
            return None
        return [_exact_rot(c, s["q"], s["pos"]), _exact_stored(c, _exact_rot(c, s["k"], s["pos"])),
                _exact_stored(c, s["v"].double())]
    if c["op"] == "keep":
        return None
    B, T, H, Hkv, hd, page = c["B"], c["T"], c["H"], c["Hkv"], c["hd"], c["page"]
    out = torch.zeros(B, T, H, hd, dtype=torch.float64, device=DEV)
    lse = torch.full((B, T, H), -math.inf, dtype=torch.float64, device=DEV)
    for b in range(B):
        P, n = int(s["start"][b]), int(s["nodes"][b])
        at = torch.arange(P + n, device=DEV)
        see = torch.ones(n, P + n, dtype=torch.bool, device=DEV)
        see[:, P:] = torch.ones(n, n, device=DEV).tril().bool() if s["mask"] is None else s["mask"][b, :n, :n].bool()
        for h in range(Hkv):
            kv = []
            for name in ("k", "v"):
                x = s[name + "_cache"][0]
                x = x[s["table"][b].long()[at // page], h, at % page] if page else x[b, h, at]
                x = x.double()
                if c["cache"] == "e4m3":
                    z = s[name + "_scale"][0]
                    z = z[s["table"][b].long()[at // page], h, at % page] if page else z[b, h, at]
                    x = x * z.double()[:, None]
                kv.append(x)
            G = H // Hkv
            q = s["q"][b, :n, h * G:(h + 1) * G].double().transpose(0, 1)
            x = (q @ kv[0].T / math.sqrt(hd)).masked_fill(~see, -math.inf)
            z = torch.logsumexp(x, -1)
            out[b, :n, h * G:(h + 1) * G] = (torch.exp(x - z[..., None]) @ kv[1]).transpose(0, 1)
            lse[b, :n, h * G:(h + 1) * G] = z.transpose(0, 1)
    return [out, lse]
