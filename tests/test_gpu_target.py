"""The target-side operators on the GPU against plain 64-bit forms: rotary positions, the
cache's write, read and accepted-row moves, and attention of a draft tree over the cache.

Tolerances are error bounds, not fits. u is the unit roundoff of the output type
(2^-8 bfloat16, whose significand has 8 bits; 2^-24 float32):
  rotation   the table's rounding, two products and a sum in float32: 4 * 2^-24 of amplitude *
             (|a| + |b|), plus u |y| for the result's rounding
  attention  scores: hd + 4 float32 roundings of sum |q k| scale =: A, so every probability
             carries a relative error below e = 2 (hd + 4) 2^-24 A + 2^-20 (2^x and the sums);
             the tensor-core path rounds probabilities to bfloat16 once more (2^-8).
             |d out| <= (e + that) sum p |v| + u |out|, |d lse| <= e + 2^-23 |lse|
"""
import math

import pytest
import torch

import target_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fe():
    import paper_2509_20416_gb300 as fe
    return fe


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rows(g, dtype, B, T, heads, hd, how="fused"):
    """Rows as a user holds them: a slice of a fused projection (16-byte aligned strides), a
    head-major view, or a view off the 16-byte grid."""
    dt = ref.DT[dtype]
    if how == "fused":
        x = torch.randn(B, T, heads + 3, hd, generator=g).to(dt).cuda()
        return x[:, :, 1:heads + 1]
    if how == "heads":
        return torch.randn(B, heads, T, hd, generator=g).to(dt).cuda().transpose(1, 2)
    x = torch.randn(B * T * heads * (hd + 1) + 1, generator=g).to(dt).cuda()
    return x[1:].view(B, T, heads, hd + 1)[..., :hd]


SCALED = dict(rope_factor=4.0, rope_orig=128.0)


# ---- rotary positions --------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("hd,rd,how", [(128, 128, "fused"), (128, 64, "heads"), (64, 64, "odd"), (64, 48, "fused"),
                                       (128, 6, "fused"), (64, 20, "odd"), (128, 2, "heads")])
@pytest.mark.parametrize("backward", [False, True])
def test_rope(fe, dtype, layout, hd, rd, how, backward):
    c = ref.config(head_dim=hd, rope_dim=rd, rope_layout=layout, dtype=dtype, n_heads=5, n_kv_heads=1, max_batch=3,
                   max_seq=4000)
    t = fe.fe_target_init(c)
    g = gen(7)
    for T in (1, 37):
        q, k = rows(g, dtype, 3, T, 5, hd, how), rows(g, dtype, 3, T, 1, hd, how)
        pos = torch.randint(0, 4000, (3, T), generator=g, dtype=torch.int32)
        pos[0, 0], pos[-1, -1] = 0, 3999
        pos = pos.cuda()
        qo, ko = fe.fe_rope(t, q, k, pos, backward=backward)
        q2 = q.clone(memory_format=torch.preserve_format) if how == "heads" else q
        want = [ref.rotate(c, x, pos, backward) for x in (q, k)]
        fe.fe_rope(t, q2, None, pos, backward=backward, q_out=q2)  # in place
        assert torch.equal(q2, qo)
        for got, (y, mag) in zip((qo, ko), want):
            tol = 4 * 2.0 ** -24 * mag + ref.UNIT[dtype] * y.abs() + 1e-30
            assert ((got.double() - y).abs() <= tol).all()
    assert fe.fe_target_status(t) == fe.FE_OK


@pytest.mark.parametrize("scaling,extra", [("none", {}), ("linear", {}), ("ntk", {}),
                                           ("bands", dict(rope_low=1.0, rope_high=4.0)),
                                           ("yarn", dict(rope_low=8.0, rope_high=1.0))])
def test_rope_scalings_and_long_positions(fe, scaling, extra):
    c = ref.config(dtype="f32", n_heads=2, n_kv_heads=2, head_dim=64, max_batch=1, max_seq=1 << 20, rope_theta=5e5,
                   rope_scaling=scaling, **SCALED, **extra)
    t = fe.fe_target_init(c)
    g = gen(3)
    q = torch.randn(1, 64, 2, 64, generator=g).cuda()
    pos = torch.randint(0, 1 << 20, (1, 64), generator=g, dtype=torch.int32).cuda()
    pos[0, 0] = (1 << 20) - 1
    got, _ = fe.fe_rope(t, q, None, pos)
    y, mag = ref.rotate(c, q, pos)
    # a float64 angle of 2^20 radians is itself off by up to 2^-33: below the float32 bound
    assert ((got.double() - y).abs() <= 4 * 2.0 ** -24 * mag).all()


def test_rope_gradient_is_the_transpose(fe):
    """<g, R x> = <R' g, x>, and differences of the forward map along random directions."""
    c = ref.config(dtype="f32", n_heads=4, n_kv_heads=2, rope_dim=96, rope_scaling="yarn", rope_low=8.0, rope_high=1.0,
                   **SCALED)
    t = fe.fe_target_init(c)
    g = gen(11)
    x, go, dx = (torch.randn(2, 19, 4, 128, generator=g).cuda() for _ in range(3))
    pos = torch.randint(0, 512, (2, 19), generator=g, dtype=torch.int32).cuda()
    fwd = lambda z: fe.fe_rope(t, z, None, pos)[0].double()
    back = fe.fe_rope(t, go, None, pos, backward=True)[0].double()
    n = x.numel()
    # each of n products of numbers of size ~1..4 is off by at most 8 * 2^-24 * 4
    tol = n * 32 * 2.0 ** -24
    assert abs((go.double() * fwd(x)).sum() - (back * x.double()).sum()).item() < tol
    h = 0.5
    diff = (fwd(x + h * dx) - fwd(x - h * dx)) / (2 * h)
    assert abs((go.double() * diff).sum() - (back * dx.double()).sum()).item() < 4 * tol


def test_rope_positions_out_of_range_leave_the_row(fe):
    c = ref.config(max_seq=100)
    t = fe.fe_target_init(c)
    q = torch.randn(1, 4, 8, 128, generator=gen(1)).bfloat16().cuda()
    pos = torch.tensor([[5, 100, -1, 99]], dtype=torch.int32).cuda()
    out = torch.full_like(q, 7.0)
    fe.fe_rope(t, q, None, pos, q_out=out)
    assert fe.fe_target_status(t) == fe.FE_ERR_CAPACITY
    assert fe.fe_target_status(t) == fe.FE_OK  # cleared
    assert (out[0, 1:3] == 7.0).all() and (out[0, 0] != 7.0).any() and (out[0, 3] != 7.0).any()


# ---- the cache -------------------------------------------------------------------------------------


def slots_of(c, x, b, table):
    """All max_seq slots of sequence b as [max_seq, Hkv, ...]."""
    ps = c["page_size"]
    if not ps:
        return x[b].transpose(0, 1)
    at = torch.arange(c["max_seq"], device=x.device)
    return x[table[b].long()[at // ps], :, at % ps]


@pytest.mark.parametrize("dtype,cache", [("bf16", "e4m3"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("hd,page,how,rot", [(128, 0, "fused", True), (64, 16, "odd", True), (128, 5, "heads", False),
                                             (64, 1, "fused", False), (128, 24, "odd", False)])
def test_cache_write_and_read(fe, dtype, cache, hd, page, how, rot):
    c = ref.config(dtype=dtype, cache_dtype=cache, head_dim=hd, page_size=page, n_heads=6, n_kv_heads=3, max_batch=3,
                   max_seq=90, rope_dim=hd // 2)
    t = fe.fe_target_init(c)
    g = gen(hd + page)
    table, n_pages = ref.paged(c, 3, g)
    store = ref.random_cache(fe, t, c, g, layers=2, table=table, n_pages=n_pages)
    before = [x.clone().view(torch.uint8) for x in (store.k, store.v)]
    T = 21
    k, v = rows(g, dtype, 3, T, 3, hd, how), rows(g, dtype, 3, T, 3, hd, how)
    q = rows(g, dtype, 3, T, 6, hd, how)
    v[0, 0, 0], v[1, 2, 1] = 0.0, v[1, 2, 1] * 1e-30
    start = torch.tensor([0, 33, 69], dtype=torch.int32).cuda()
    n_rows = torch.tensor([T, 0 + 13, T], dtype=torch.int32).cuda()
    pos = (start[:, None] + torch.arange(T, device="cuda", dtype=torch.int32) // 2).contiguous() if rot else None
    qo = fe.fe_cache_write(t, store, 1, k, v, start, n_rows=n_rows, pos=pos, q=q if rot else None)
    ko, vo = fe.fe_cache_read(t, store, 1, start, n_rows, T + 2)
    assert fe.fe_target_status(t) == fe.FE_OK
    if rot:
        assert torch.equal(qo, fe.fe_rope(t, q, None, pos)[0])
    for x, want, old, sc, back, rotated in ((store.k, k, before[0], store.k_scale, ko, rot),
                                            (store.v, v, before[1], store.v_scale, vo, False)):
        assert torch.equal(x[0].view(torch.uint8), old[0])  # the other layer
        y, mag = ref.rotate(c, want, pos) if rotated else (want.double(), want.double().abs())
        for b in range(3):
            n, s0 = int(n_rows[b]), int(start[b])
            now = slots_of(c, x[1], b, table)
            was = slots_of(c, old[1].view(x.dtype), b, table)
            free = torch.ones(c["max_seq"], dtype=torch.bool)
            free[s0:s0 + n] = False
            assert torch.equal(now.view(torch.uint8)[free], was.view(torch.uint8)[free])
            got, exact = now[s0:s0 + n].double(), y[b, :n]
            assert (back[b, n:] == 0).all()
            if cache == "e4m3":
                scale = slots_of(c, sc[1], b, table)[s0:s0 + n].double()
                e, s = ref.quantise(exact)
                if rotated:  # float32 rotation: a value next to a rounding boundary may go either way
                    assert ((scale == s) | (scale == 2 * s) | (scale == s / 2)).all()
                    # half a step of e4m3: 2^-4 of the value, or 2^-10 of the scale below 2^-6
                    tol = torch.maximum(exact.abs() / 16, scale[..., None] * 2.0 ** -10) + 4 * 2.0 ** -24 * mag[b, :n]
                    assert ((got * scale[..., None] - exact).abs() <= tol * (1 + 1e-6)).all()
                else:
                    assert torch.equal(got, e) and torch.equal(scale, s)
                assert torch.equal(back[b, :n].double(), got * scale[..., None])
            else:
                tol = 4 * 2.0 ** -24 * mag[b, :n] + ref.UNIT[dtype] * exact.abs() if rotated else 0.0 * exact
                assert ((got - exact).abs() <= tol).all()
                assert torch.equal(back[b, :n], now[s0:s0 + n])


def test_cache_quantisation_edges(fe):
    """Zeros, the smallest and largest scales, ties, subnormals and non-finite elements."""
    c = ref.config(cache_dtype="e4m3", n_heads=1, n_kv_heads=1, max_batch=1, max_seq=16)
    t = fe.fe_target_init(c)
    store = fe.alloc_cache(t, 1)
    x = torch.randn(1, 10, 1, 128, generator=gen(5))
    x[0, 0] = 0.0
    x[0, 1] *= 2.0 ** -126
    x[0, 2] *= 2.0 ** 120
    x[0, 3] = torch.arange(128) / 16.0  # ties between neighbours
    x[0, 3, 0, 0] = 448.0
    x[0, 4] = 448.0 * 2.0 ** -torch.arange(128.0).clamp(max=40)
    x[0, 5, 0, 3], x[0, 5, 0, 4], x[0, 5, 0, 5] = math.nan, math.inf, -math.inf
    x[0, 6] = math.inf
    x[0, 7, 0, 0] = 450.0  # (bfloat16 450: just above 448)
    x = x.bfloat16().cuda()
    start, n = torch.zeros(1, dtype=torch.int32).cuda(), torch.full((1,), 10, dtype=torch.int32).cuda()
    fe.fe_cache_write(t, store, 0, x, x, start)
    e, s = ref.quantise(x[0, :, 0])
    got, scale = store.k[0, 0, 0, :10].double(), store.k_scale[0, 0, 0, :10].double()
    assert torch.equal(scale, s)
    assert torch.equal(torch.isnan(got), torch.isnan(e)) and torch.equal(got.nan_to_num(0), e.nan_to_num(0))
    ko, vo = fe.fe_cache_read(t, store, 0, start, n, 10)
    assert torch.equal(torch.isnan(ko[0, :, 0]), torch.isnan(e))
    want = (e * s[:, None]).to(torch.bfloat16).double()
    assert torch.equal(ko[0, :, 0].double().nan_to_num(0), want.nan_to_num(0)) and torch.equal(ko.nan_to_num(0), vo.nan_to_num(0))
    assert fe.fe_target_status(t) == fe.FE_OK


@pytest.mark.parametrize("page", [0, 8])
def test_cache_rows_out_of_range_are_skipped(fe, page):
    c = ref.config(page_size=page, max_seq=40, n_heads=2, n_kv_heads=2)
    t = fe.fe_target_init(c)
    g = gen(2)
    table, n_pages = ref.paged(c, 2, g)
    store = ref.random_cache(fe, t, c, g, table=table, n_pages=n_pages)
    old = store.k.clone()
    k = rows(g, "bf16", 2, 6, 2, 128)
    for start in ([36, 2**31 - 1], [-3, 40]):
        s = torch.tensor(start, dtype=torch.int32).cuda()
        fe.fe_cache_write(t, store, 0, k, k, s)
        assert fe.fe_target_status(t) == fe.FE_ERR_CAPACITY
    now = slots_of(c, store.k[0], 0, table)
    was = slots_of(c, old[0], 0, table)
    assert torch.equal(now[36:40], k[0, :4]) and torch.equal(now[:3], k[0, 3:]) and torch.equal(now[3:36], was[3:36])
    assert torch.equal(slots_of(c, store.k[0], 1, table), slots_of(c, old[0], 1, table))
    s, n = torch.tensor([38, 0], dtype=torch.int32).cuda(), torch.tensor([4, 1], dtype=torch.int32).cuda()
    ko, _ = fe.fe_cache_read(t, store, 0, s, n, 4)
    assert fe.fe_target_status(t) == fe.FE_ERR_CAPACITY
    assert (ko[0, 2:] == 0).all() and torch.equal(ko[0, :2], now[38:]) and (ko[1, 1:] == 0).all()
    if page:
        table[0, 1] = n_pages
        fe.fe_cache_read(t, store, 0, torch.tensor([8, 0], dtype=torch.int32).cuda(), n, 4)
        assert fe.fe_target_status(t) == fe.FE_ERR_DEVICE


@pytest.mark.parametrize("dtype,cache,hd", [("bf16", "e4m3", 128), ("bf16", "bf16", 64), ("f32", "f32", 128), ("bf16", "e4m3", 64)])
@pytest.mark.parametrize("page", [0, 4])
def test_cache_keep(fe, dtype, cache, hd, page):
    c = ref.config(dtype=dtype, cache_dtype=cache, head_dim=hd, page_size=page, n_heads=3, n_kv_heads=3, max_batch=5,
                   max_seq=64)
    t = fe.fe_target_init(c)
    g = gen(page + hd)
    table, n_pages = ref.paged(c, 5, g)
    store = ref.random_cache(fe, t, c, g, layers=131, table=table, n_pages=n_pages)
    path = torch.tensor([[1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11], [2, 3, 5, 8, 9, 20, 21, 22, 30, 31, 33],
                         [40, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0], [-1] * 11, [3, 9, 10, 11, 12, 30, 31, 32, 33, 50, 52]],
                        dtype=torch.int32)
    n = torch.tensor([11, 11, 1, 0, 9], dtype=torch.int32)
    start = torch.tensor([0, 30, 23, 5, 11], dtype=torch.int32)
    old = {m: getattr(store, m).clone() for m in ("k", "v", "k_scale", "v_scale") if getattr(store, m) is not None}
    fe.fe_cache_keep(t, store, path.cuda(), n.cuda(), start.cuda())
    assert fe.fe_target_status(t) == fe.FE_OK
    raw = lambda x: x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
    for m, was in old.items():
        now = getattr(store, m)
        for layer in (0, 1, 127, 130):
            for b in range(5):
                want, got = slots_of(c, raw(was[layer]), b, table).clone(), slots_of(c, raw(now[layer]), b, table)
                src = slots_of(c, raw(was[layer]), b, table)
                for j in range(int(n[b])):
                    want[start[b] + 1 + j] = src[start[b] + path[b, j]]
                assert torch.equal(got, want), (m, layer, b)


@pytest.mark.parametrize("path,n,start,code", [([[2, 2]], 2, 0, "DEVICE"), ([[0, 1]], 2, 0, "DEVICE"), ([[3, 1]], 2, 0, "DEVICE"),
                                               ([[1, 3]], 3, 0, "DEVICE"), ([[1, 3]], -1, 0, "DEVICE"),
                                               ([[1, 30]], 2, 40, "CAPACITY"), ([[1, 2]], 2, -5, "CAPACITY")])
def test_cache_keep_refuses_bad_paths(fe, path, n, start, code):
    c = ref.config(max_seq=64, max_batch=1)
    t = fe.fe_target_init(c)
    store = ref.random_cache(fe, t, c, gen(1))
    old = store.k.clone()
    i = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    fe.fe_cache_keep(t, store, i(path), i([n]), i([start]))
    assert fe.fe_target_status(t) == getattr(fe, "FE_ERR_" + code)
    assert torch.equal(store.k, old)


# ---- attention ------------------------------------------------------------------------------------


def tree_masks(g, B, T):
    """Random trees' ancestor-or-self masks."""
    m = torch.zeros(B, T, T, dtype=torch.uint8)
    for b in range(B):
        for i in range(T):
            if i:
                m[b, i] = m[b, int(torch.randint(max(0, i - 9), i, (1,), generator=g))]
            m[b, i, i] = 1
    return m


def check_attention(c, store, table, q, P, n, mask, out, lse, scale=None, heads=None):
    H, Hkv, hd = c["n_heads"], c["n_kv_heads"], c["head_dim"]
    G, T = H // Hkv, q.shape[1]
    scale = 1 / math.sqrt(hd) if scale is None else scale
    rounding = 0.0 if c["dtype"] == "f32" else ref.UNIT["bf16"]
    for b in range(q.shape[0]):
        nb = int(n[b])
        assert (out[b, nb:] == 0).all() and (lse[b, nb:] == -math.inf).all()
        if nb == 0:
            continue
        see = torch.ones(nb, int(P[b]) + nb, dtype=torch.bool, device="cuda")
        see[:, int(P[b]):] = (mask[b, :nb, :nb].cuda() != 0) if mask is not None else torch.ones(nb, nb, device="cuda").tril().bool()
        for h in (range(Hkv) if heads is None else heads):
            k, v = ref.cache_rows(c, store, 0, b, h, int(P[b]) + nb, table)
            for gq in range(G):
                o, l, size, A = ref.attend(q[b, :nb, h * G + gq], k, v, see, scale)
                e = (2 * (hd + 4) * 2.0 ** -24 * A + 2.0 ** -20)[:, None]
                got, gl = out[b, :nb, h * G + gq].double(), lse[b, :nb, h * G + gq].double()
                fin = torch.isfinite(o)
                assert torch.equal(torch.isfinite(got), fin), (b, h, gq)
                tol = (e + 1.01 * rounding) * size + ref.UNIT[c["dtype"]] * o.abs() + 1e-30
                bad = ((got - o).abs() > tol) & fin
                assert not bad.any(), (b, h, gq, float(((got - o).abs() / tol)[fin].max()))
                empty = l == -math.inf
                assert torch.equal(gl == -math.inf, empty)
                ok = ((gl - l).abs() <= e[:, 0] + 2.0 ** -23 * l.abs()) | empty | ~torch.isfinite(l)
                assert ok.all(), (b, h, gq, float((gl - l).abs().max()))


SHAPES = [  # H, Hkv, hd, T, prefixes, page, mask, ragged
    (4, 4, 64, 1, [0, 1, 63, 64], 0, "causal", False),
    (32, 8, 128, 1, [199, 0, 127, 128], 16, "causal", False),
    (8, 2, 128, 11, [5, 700], 0, "tree", False),
    (8, 1, 128, 49, [256, 0, 333], 16, "tree", True),
    (64, 8, 128, 81, [130], 0, "tree", False),
    (5, 5, 64, 130, [100, 1], 5, "tree", True),
    (6, 2, 128, 257, [17, 380], 24, "causal", True),
    (12, 4, 64, 200, [0, 9], 1, "causal", False),
    (3, 3, 128, 7, [1500], 0, "tree", False),
    (16, 1, 64, 40, [250, 251, 252, 0, 3], 64, "tree", True),
]


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x) for x in s))
def test_tree_attention(fe, dtype, cache, shape):
    H, Hkv, hd, T, P, page, kind, ragged = shape
    B = len(P)
    c = ref.config(dtype=dtype, cache_dtype=cache, n_heads=H, n_kv_heads=Hkv, head_dim=hd, page_size=page, max_batch=B,
                   max_seq=max(P) + T + 3)
    t = fe.fe_target_init(c)
    g = gen(T + hd)
    table, n_pages = ref.paged(c, B, g)
    store = ref.random_cache(fe, t, c, g, table=table, n_pages=n_pages)
    q = rows(g, dtype, B, T, H, hd, "heads" if page == 5 else "odd" if page == 1 else "fused") * 2
    n = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32) if ragged else torch.full((B,), T, dtype=torch.int32)
    if ragged:
        n[0] = T
    mask = tree_masks(g, B, T) if kind == "tree" else None
    plen = torch.tensor(P, dtype=torch.int32)
    args = (t, store, 0, q, plen.cuda())
    kw = dict(mask=None if mask is None else mask.cuda(), n_nodes=n.cuda() if ragged else None)
    out, lse = fe.fe_tree_attention(*args, **kw)
    assert fe.fe_target_status(t) == fe.FE_OK
    check_attention(c, store, table, q, plen, n, mask, out, lse)
    out2, lse2 = fe.fe_tree_attention(*args, **kw)
    assert torch.equal(out.view(torch.uint8), out2.view(torch.uint8)) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("T,P", [(9, [0, 3]), (40, [120, 260]), (140, [0, 700])])
def test_hidden_slots_do_not_matter(fe, dtype, cache, T, P):
    """Rows that see nothing, NaN and infinities in slots that a node does not see (other
    branches, slots past the tree), and in one that some nodes do see."""
    B, H, Hkv, hd = len(P), 6, 2, 128
    c = ref.config(dtype=dtype, cache_dtype=cache, n_heads=H, n_kv_heads=Hkv, head_dim=hd, max_batch=B, max_seq=max(P) + T + 200)
    t = fe.fe_target_init(c)
    g = gen(T)
    store = ref.random_cache(fe, t, c, g)
    mask = tree_masks(g, B, T)
    mask[:, T // 2] = 0  # a node that sees no node
    mask[:, :, 2] = 0
    mask[:, 2, 2] = 1
    odd = [T - 1, T - 3, 2]
    mask[:, T - 1, :] = 0  # its own row holds NaN: hidden from everyone, itself included
    mask[:, :, T - 1] = 0
    n = torch.full((B,), T, dtype=torch.int32)
    for b in range(B):
        for x in (store.k, store.v):
            x[0, b, :, P[b] + T:] = math.nan
            x[0, b, :, P[b] + odd[0]] = math.nan
        if cache == "e4m3":
            store.v[0, b, 0, P[b] + odd[1], 5] = math.nan
            store.v_scale[0, b, :, P[b] + T:] = math.nan
        else:
            store.v[0, b, 0, P[b] + odd[1], 5] = math.inf
            store.v[0, b, 1, P[b] + odd[2], 100] = -math.inf
            store.k[0, b, 1, P[b] + odd[1], 9] = math.nan
    q = rows(g, dtype, B, T, H, hd)
    plen = torch.tensor(P, dtype=torch.int32)
    out, lse = fe.fe_tree_attention(t, store, 0, q, plen.cuda(), mask=mask.cuda())
    assert fe.fe_target_status(t) == fe.FE_OK
    assert torch.isnan(out).any(-1).any() or torch.isinf(out).any()
    check_attention(c, store, None, q, plen, n, mask, out, lse)


@pytest.mark.parametrize("page", [0, 3, 16, 128, 256])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "e4m3")])
def test_what_lies_past_the_end_does_not_matter(fe, dtype, cache, causal, page):
    """Slots from P + n on and the pool's other pages may hold anything, their page ids too."""
    B, T, H, Hkv, P, ragged = 4, 150, 8, 4, (0, 100, 129, 511), (150, 3, 127, 0)
    c = ref.config(dtype=dtype, cache_dtype=cache, n_heads=H, n_kv_heads=Hkv, head_dim=64, page_size=page, max_batch=B, max_seq=896)
    t = fe.fe_target_init(c)
    g = gen(page)
    table, n_pages = ref.paged(c, B, g)
    store = ref.random_cache(fe, t, c, g, table=table, n_pages=n_pages)
    q, mask = rows(g, dtype, B, T, H, 64), None if causal else tree_masks(g, B, T).cuda()
    plen, n = torch.tensor(P, dtype=torch.int32).cuda(), torch.tensor(ragged, dtype=torch.int32).cuda()
    want = fe.fe_tree_attention(t, store, 0, q, plen, n_nodes=n, mask=mask)
    kept = [x[0].clone() for x in (store.k, store.v, store.k_scale, store.v_scale) if x is not None]
    for x, y in zip([x[0] for x in (store.k, store.v, store.k_scale, store.v_scale) if x is not None], kept):
        x.fill_(math.nan)
        for b in range(B):
            end = P[b] + ragged[b]
            if not page:
                x[b, :, :end] = y[b, :, :end]
                continue
            for s in range(0, end, page):
                pg, rows_ = int(table[b, s // page]), min(page, end - s)
                x[pg, :, :rows_] = y[pg, :, :rows_]
    if page:
        for b in range(B):
            table[b, (P[b] + ragged[b] + page - 1) // page:] = -7
    got = fe.fe_tree_attention(t, store, 0, q, plen, n_nodes=n, mask=mask)
    assert fe.fe_target_status(t) == fe.FE_OK
    assert torch.isfinite(want[0]).all() and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("scale", [math.nan, math.inf, -math.inf, 0.0, 3e38, -1.0, 1e-40])
def test_hidden_rows_with_any_scale(fe, scale):
    """A row that no node sees may hold any scale: branches whose rows were never written."""
    B, T, H, Hkv, hd, P = 2, 40, 8, 2, 128, (129, 700)
    c = ref.config(dtype="bf16", cache_dtype="e4m3", n_heads=H, n_kv_heads=Hkv, head_dim=hd, max_batch=B, max_seq=800)
    t = fe.fe_target_init(c)
    g = gen(T)
    store = ref.random_cache(fe, t, c, g)
    mask = tree_masks(g, B, T)
    mask[:, 5, :] = 0
    mask[:, :, 5] = 0
    n = torch.full((B,), T, dtype=torch.int32)
    q = rows(g, "bf16", B, T, H, hd)
    plen = torch.tensor(P, dtype=torch.int32)
    want = fe.fe_tree_attention(t, store, 0, q, plen.cuda(), mask=mask.cuda())
    for b in range(B):
        store.k_scale[0, b, :, P[b] + 5] = scale
        store.v_scale[0, b, :, P[b] + 5] = scale
    got = fe.fe_tree_attention(t, store, 0, q, plen.cuda(), mask=mask.cuda())
    assert fe.fe_target_status(t) == fe.FE_OK
    assert torch.isfinite(want[0]).all() and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "e4m3")])
def test_attention_score_ranges(fe, dtype, cache):
    """Scores far apart (one slot takes all), all alike, very negative, and a growing maximum."""
    B, T, H, Hkv, hd, P = 1, 8, 4, 2, 128, 900
    c = ref.config(dtype=dtype, cache_dtype=cache, n_heads=H, n_kv_heads=Hkv, head_dim=hd, max_batch=B, max_seq=1024)
    t = fe.fe_target_init(c)
    for seed, (qs, kind) in enumerate([(60.0, "wide"), (0.0, "alike"), (30.0, "negative"), (30.0, "growing")]):
        g = gen(seed)
        store = ref.random_cache(fe, t, c, g)
        q = torch.randn(B, T, H, hd, generator=g) * qs
        if kind in ("negative", "growing"):
            d = torch.randn(hd, generator=g)
            q = (q * 0.02 + d * 2).expand(B, T, H, hd)
            ramp = -torch.ones(1024) * 8 if kind == "negative" else torch.linspace(-8, 8, 1024)
            k = (ramp[:, None] * d)[None, None].expand(B, Hkv, 1024, hd).to(torch.bfloat16).float()
            if cache == "e4m3":
                e, s = ref.quantise(k)
                store.k[0].copy_(e.to(torch.float8_e4m3fn).cuda())
                store.k_scale[0].copy_(s.float().cuda())
            else:
                store.k[0].copy_(k.cuda())
        q = q.to(ref.DT[dtype]).cuda()
        plen = torch.tensor([P], dtype=torch.int32)
        out, lse = fe.fe_tree_attention(t, store, 0, q, plen.cuda())
        check_attention(c, store, None, q, plen, torch.tensor([T]), None, out, lse)


@pytest.mark.parametrize("T,P", [(5, 300), (70, 300)])
def test_attention_over_e4m3_of_every_scale(fe, T, P):
    """Value and key rows of very large and very small scale (factors beyond one bfloat16 multiply),
    NaN numbers in the prefix, queries of every size and a NaN query."""
    B, H, Hkv, hd = 1, 6, 2, 128
    c = ref.config(cache_dtype="e4m3", n_heads=H, n_kv_heads=Hkv, head_dim=hd, max_batch=B, max_seq=P + T + 1)
    t = fe.fe_target_init(c)
    g = gen(T)
    store = ref.random_cache(fe, t, c, g)
    for h, shift in ((0, 12), (1, -60)):  # one head's rows far above 2^7, one's far below
        store.v_scale[0, 0, h] *= 2.0 ** shift
        store.k_scale[0, 0, h] *= 2.0 ** (-shift)
    store.v_scale[0, 0, 1, 40:60] *= 2.0 ** 30
    q = torch.randn(B, T, H, hd, generator=g)
    q[:, :, :3] *= 2.0 ** 12
    q[:, :, 3:] *= 2.0 ** -60
    q[:, 1] *= 0.0
    q = q.to(torch.bfloat16).cuda()
    plen, n = torch.tensor([P], dtype=torch.int32), torch.tensor([T])
    out, lse = fe.fe_tree_attention(t, store, 0, q, plen.cuda())
    check_attention(c, store, None, q, plen, n, None, out, lse)
    store.v[0, 0, 0, 7, 11] = math.nan
    q[0, 2, 4, 9] = math.nan
    out2, lse2 = fe.fe_tree_attention(t, store, 0, q, plen.cuda())
    assert torch.isnan(out2[:, :, :3, 11]).all() and torch.isnan(out2[0, 2, 4]).all() and torch.isnan(lse2[0, 2, 4])
    same = torch.ones_like(out2, dtype=torch.bool)
    same[:, :, :3, 11] = False
    same[0, 2, 4] = False
    assert torch.equal(out2[same], out[same])
    assert fe.fe_target_status(t) == fe.FE_OK


def test_attention_strided_output_scale_and_stream(fe):
    c = ref.config(max_batch=2, max_seq=600, page_size=16, cache_dtype="e4m3")
    t = fe.fe_target_init(c)
    g = gen(9)
    table, n_pages = ref.paged(c, 2, g)
    store = ref.random_cache(fe, t, c, g, table=table, n_pages=n_pages)
    q = rows(g, "bf16", 2, 33, 8, 128)
    plen = torch.tensor([500, 80], dtype=torch.int32)
    n = torch.tensor([33, 33])
    big = torch.full((2, 8, 33, 129), 5.0, dtype=torch.bfloat16, device="cuda")
    view = big[..., 1:].transpose(1, 2)  # off the 16-byte grid, head-major
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out, lse = fe.fe_tree_attention(t, store, 0, q, plen.cuda(), scale=0.3, out=view, stream=s)
    assert fe.fe_target_status(t, stream=s) == fe.FE_OK
    check_attention(c, store, table, q, plen, n, None, out, lse, scale=0.3)
    assert (big[..., 0] == 5.0).all()


def test_attention_lengths_out_of_range(fe):
    c = ref.config(max_batch=4, max_seq=64)
    t = fe.fe_target_init(c)
    store = ref.random_cache(fe, t, c, gen(1))
    q = rows(gen(2), "bf16", 4, 5, 8, 128)
    plen = torch.tensor([60, -1, 2**31 - 3, 10], dtype=torch.int32)
    out, lse = fe.fe_tree_attention(t, store, 0, q, plen.cuda())
    assert fe.fe_target_status(t) == fe.FE_ERR_CAPACITY
    check_attention(c, store, None, q, plen, torch.tensor([0, 0, 0, 5]), None, out, lse)
    n = torch.tensor([4, 6, -1, 0], dtype=torch.int32)
    plen = torch.tensor([60, 2, 2, 2], dtype=torch.int32)
    out, lse = fe.fe_tree_attention(t, store, 0, q, plen.cuda(), n_nodes=n.cuda())
    assert fe.fe_target_status(t) == fe.FE_ERR_CAPACITY
    check_attention(c, store, None, q, plen, torch.tensor([4, 0, 0, 0]), None, out, lse)


def test_attention_bad_page_is_reported(fe):
    c = ref.config(page_size=16, max_seq=256, max_batch=1)
    t = fe.fe_target_init(c)
    g = gen(4)
    table, n_pages = ref.paged(c, 1, g)
    store = ref.random_cache(fe, t, c, g, table=table, n_pages=n_pages)
    q = rows(g, "bf16", 1, 3, 8, 128)
    for bad in (-1, n_pages):
        table[0, 3] = bad
        out, _ = fe.fe_tree_attention(t, store, 0, q, torch.tensor([100], dtype=torch.int32).cuda())
        assert fe.fe_target_status(t) == fe.FE_ERR_DEVICE
        assert torch.isfinite(out).all()


def test_cache_past_32_bit_offsets(fe):
    """A cache of more than 2^32 elements: the last sequence's last head lies past every 32-bit
    byte and element offset."""
    c = ref.config(cache_dtype="e4m3", n_heads=4, n_kv_heads=4, max_batch=9, max_seq=1 << 20, rope_theta=5e5)
    t = fe.fe_target_init(c)
    store = fe.alloc_cache(t, 1)
    assert store.k.numel() > 1 << 32
    g = gen(6)
    B, T = 9, 3
    P = [0] * 8 + [(1 << 20) - 3]
    plen = torch.tensor(P, dtype=torch.int32).cuda()
    near = torch.tensor([0] * 8 + [(1 << 20) - 300], dtype=torch.int32).cuda()
    k, v = (torch.randn(B, 300, 4, 128, generator=g).bfloat16().cuda() for _ in range(2))
    fe.fe_cache_write(t, store, 0, k, v, near)
    q = torch.randn(B, T, 4, 128, generator=g).bfloat16().cuda()
    out, lse = fe.fe_tree_attention(t, store, 0, q, plen)
    ko, vo = fe.fe_cache_read(t, store, 0, near, torch.full((B,), 300, dtype=torch.int32).cuda(), 300)
    assert fe.fe_target_status(t) == fe.FE_OK
    e, s = ref.quantise(k)
    assert torch.equal(ko.double(), e * s[..., None])
    for i in range(T):
        n = (1 << 20) - 3 + i + 1
        for h in (0, 3):
            x = (store.k[0, 8, h, :n].float() * store.k_scale[0, 8, h, :n, None]).double() @ q[8, i, h].double() / math.sqrt(128)
            want = torch.softmax(x, 0) @ (store.v[0, 8, h, :n].float() * store.v_scale[0, 8, h, :n, None]).double()
            assert abs(torch.logsumexp(x, 0) - lse[8, i, h].double()) < 1e-4
            assert (out[8, i, h].double() - want).abs().max() <= 2.0 ** -8 * want.abs().max() + 1e-7
    path, acc = torch.tensor([[2]] * 9, dtype=torch.int32).cuda(), torch.tensor([0] * 8 + [1], dtype=torch.int32).cuda()
    last = store.k[0, 8, 3, -1].clone()
    fe.fe_cache_keep(t, store, path, acc, plen)
    assert torch.equal(store.k[0, 8, 3, -2].view(torch.uint8), last.view(torch.uint8))


def test_calls_refuse_bad_arguments(fe):
    from paper_2509_20416_gb300 import target as tg
    c = ref.config(max_seq=64, cache_dtype="e4m3")
    t = fe.fe_target_init(c)
    store = fe.alloc_cache(t, 1)
    q, k = rows(gen(1), "bf16", 2, 4, 8, 128), rows(gen(2), "bf16", 2, 4, 2, 128)
    i = torch.zeros(2, 4, dtype=torch.int32).cuda()
    s = i[:, 0].contiguous()
    bad = [
        lambda: fe.fe_tree_attention(t, store, 0, q, s, scale=math.nan),
        lambda: fe.fe_cache_write(t, store, 0, k, k, s, q=q),  # queries without positions
        lambda: fe.fe_rope(t, None, None, i),
        lambda: fe.fe_cache_read(t, store, 0, s, s, 65),
        lambda: fe.fe_tree_attention(t, store, 0, torch.zeros(3, 1, 8, 128).bfloat16().cuda(), torch.zeros(3, dtype=torch.int32).cuda()),
    ]
    for call in bad:
        with pytest.raises(fe.FeError) as e:
            call()
        assert e.value.code == fe.FE_ERR_INVALID_ARG
    for wrong in (q.float(), q[..., :64], q[:, :, :4]):
        with pytest.raises(ValueError):
            fe.fe_tree_attention(t, store, 0, wrong, s)
    for call in (lambda: fe.fe_tree_attention(t, store, 0, q, s.long()), lambda: fe.fe_tree_attention(t, store, 1, q, s),
                 lambda: fe.fe_tree_attention(t, store, 0, q, s, mask=torch.zeros(2, 4, 5, dtype=torch.uint8).cuda()),
                 lambda: fe.fe_rope(t, q, None, i[:, :3]), lambda: fe.fe_cache_keep(t, store, i, s, i),
                 lambda: fe.Cache(t, [store.k[0, :1]], [store.v[0]], store.k_scale, store.v_scale)):
        with pytest.raises(ValueError):
            call()
    # a cache off the 16-byte grid is refused by the library itself
    rows_q = tg._rows(t, q, q.shape)
    args = tg._PACK["fe_tree_attention"](2, 4, *rows_q, *rows_q, 0, s.data_ptr(), 0, 0, 1.0, store.k.data_ptr() + 8,
                                         store.v.data_ptr(), store.k_scale.data_ptr(), store.v_scale.data_ptr(), 0, 0)
    assert fe._lib.fe_tree_attention(t.ptr, args, None) == fe.FE_ERR_INVALID_ARG
    assert fe.fe_target_status(t) == fe.FE_OK
