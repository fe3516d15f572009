"""The target-side operators in plain 64-bit form, written from their definitions
(include/fe_target.h), and the inputs that the tests share."""
import math

import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # unit roundoff: half a unit in the last place of 1


def config(**kw):
    c = dict(n_heads=8, n_kv_heads=2, head_dim=128, max_batch=2, max_seq=512, page_size=0, dtype="bf16", rope_theta=1e4)
    c.update(kw)
    return c


def freqs(c):
    rd, theta, s = c.get("rope_dim", c["head_dim"]), c["rope_theta"], c.get("rope_factor", 1.0)
    kind, L = c.get("rope_scaling", "none"), c.get("rope_orig", 0.0)
    out, amp = [], 1.0
    for i in range(rd // 2):
        b = theta ** (-2.0 * i / rd)
        if kind == "linear":
            b /= s
        elif kind == "ntk":
            b = (theta * s ** (rd / (rd - 2))) ** (-2.0 * i / rd)
        elif kind == "bands":
            turns = L * b / (2 * math.pi)
            if turns < c["rope_low"]:
                b /= s
            elif turns < c["rope_high"]:
                w = (turns - c["rope_low"]) / (c["rope_high"] - c["rope_low"])
                b = (1 - w) * b / s + w * b
        elif kind == "yarn":
            lo = max(math.floor(rd * math.log(L / (2 * math.pi * c["rope_low"])) / (2 * math.log(theta))), 0)
            hi = min(math.ceil(rd * math.log(L / (2 * math.pi * c["rope_high"])) / (2 * math.log(theta))), rd - 1)
            w = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            b = b / s * w + b * (1 - w)
            amp = 0.1 * math.log(s) + 1.0
        out.append(b)
    return torch.tensor(out, dtype=torch.float64), amp


def rotate(c, x, pos, backward=False):
    """x [B, T, heads, hd], pos [B, T] -> float64, and |a| + |b| of each element's pair."""
    f, amp = freqs(c)
    rd = c.get("rope_dim", c["head_dim"])
    x = x.double()
    y, mag = x.clone(), x.abs()
    ang = pos.double()[..., None] * f.to(x.device)
    cos, sin = amp * ang.cos()[:, :, None], amp * ang.sin()[:, :, None] * (-1 if backward else 1)
    i = torch.arange(rd // 2, device=x.device)
    a, b = (i, i + rd // 2) if c.get("rope_layout", "half") == "half" else (2 * i, 2 * i + 1)
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., a] * sin + x[..., b] * cos
    mag[..., a] = mag[..., b] = amp * (x[..., a].abs() + x[..., b].abs())
    return y, mag


def two(k):
    """2^k exactly, for whole numbers -300 < k < 300 (a 64-bit power on the GPU may be off by one
    rounding): the number's bits."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def quantise(x):
    """Rows [..., hd] -> (e4m3 values as float64, scale): the smallest 2^c, c >= -120, that
    leaves no finite element above 448; non-finite elements become NaN."""
    x = x.double()
    fin = torch.isfinite(x)
    top = torch.where(fin, x.abs(), 0.0).amax(-1)
    c = torch.full_like(top, -120.0)
    for k in range(-119, 121):
        c = torch.where(top > 448.0 * 2.0 ** (k - 1), float(k), c)
    s = two(c)
    y = torch.where(fin, x / s[..., None], math.nan)
    exp = torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent - 1
    step = two(exp - 3)
    return torch.round(y / step) * step, s


def cache_rows(c, cache, layer, b, h, n, table=None):
    """The stored rows 0 .. n - 1 of (b, h) as float64 values, and the bf16-rounded products."""
    ps = c["page_size"]
    at = torch.arange(n, device=cache.k[layer].device)
    idx = (table[b].long()[at // ps], h, at % ps) if ps else (b, h, at)
    out = []
    for x, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        r = x[layer][idx].double()
        out.append(r * s[layer][idx].double()[:, None] if s is not None else r)
    return out


def attend(q, k, v, see, scale):
    """q [R, hd], k and v [n, hd], see [R, n] -> float64 (out, lse, sum p |v|, max sum |q k|)."""
    q, k, v = q.double(), k.double(), v.double()
    s = (q[:, None] * k[None]).sum(-1) * scale
    s = torch.where(see, s, -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(s - m)
    z = p.sum(-1, keepdim=True)
    w = torch.where(z == 0, 0.0, p / z)
    # a hidden slot adds nothing, whatever it holds
    term = torch.where(see[..., None], w[..., None] * v[None], 0.0)
    size = torch.where(see, (q[:, None] * k[None]).abs().sum(-1) * abs(scale), 0.0).amax(-1)
    return term.sum(1), (m + torch.log(z))[:, 0], term.abs().sum(1), size


def paged(c, B, gen, spare=3):
    """A shuffled page table [B, pages per sequence] and the pool size (0 pages: contiguous)."""
    if not c["page_size"]:
        return None, 0
    per = -(-c["max_seq"] // c["page_size"])
    n = B * per + spare
    perm = torch.randperm(n, generator=gen)[:B * per].to(torch.int32).view(B, per)
    return perm.cuda().contiguous(), n


def random_cache(fe, t, c, gen, layers=1, table=None, n_pages=0):
    """A cache filled with random rows (quantised ones for e4m3)."""
    ps = c["page_size"]
    rows = (layers,) + ((n_pages, t.Hkv, ps) if ps else (t.max_batch, t.Hkv, t.max_seq))
    kv, sc = [], []
    for _ in range(2):
        x = torch.randn(rows + (t.hd,), generator=gen)
        if t.cache_name == "e4m3":
            y, s = quantise(x * torch.exp2(torch.randint(-3, 4, rows, generator=gen).float())[..., None])
            kv.append(y.to(torch.float8_e4m3fn).cuda())
            sc.append(s.float().cuda())
        else:
            kv.append(x.to(DT[t.cache_name]).cuda())
    return fe.Cache(t, kv[0], kv[1], *(sc if sc else (None, None)), page_table=table, n_pages=n_pages)
