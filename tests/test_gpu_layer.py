"""The dense operators of a target layer on the GPU against their 64-bit forms (layer_ref.py), within the
bounds that float32 sums and the type's roundings leave."""
import math

import pytest
import torch

import layer_ref as ref

pytestmark = pytest.mark.gpu

MARK = 77.0  # what lies around outputs


@pytest.fixture(scope="module")
def fe():
    import paper_2509_20416_gb300 as fe
    return fe


@pytest.fixture(scope="module")
def handles(fe):
    cfg = lambda dt: dict(n_heads=1, n_kv_heads=1, head_dim=64, max_seq=16, dtype=dt, rope_theta=1e4)
    return {dt: fe.fe_target_init(cfg(dt)) for dt in ("f32", "bf16")}


@pytest.fixture(autouse=True)
def no_status(fe, handles):
    yield
    for t in handles.values():
        assert fe.fe_target_status(t) == fe.FE_OK


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, dtype, *shape, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(ref.DT[dtype])


def inside(x, left=0, right=0):
    """x [R, n] as columns of a wider matrix, with `left` and `right` columns around it: other row strides and
    alignments. The wider matrix comes back too."""
    R, n = x.shape
    wide = torch.full((R + 2, left + n + right), MARK, dtype=x.dtype, device=x.device)
    wide[1:-1, left:left + n] = x
    return wide[1:-1, left:left + n], wide


def untouched(wide, left, n):
    around = wide.clone()
    around[1:-1, left:left + n] = MARK
    assert (around == MARK).all()


def both(fn, leaves, grads):
    """fn(*leaves) and the gradients of the leaves."""
    leaves = [x.detach().requires_grad_() for x in leaves]
    out = fn(*leaves)
    out = out if isinstance(out, tuple) else (out,)
    got = torch.autograd.grad([o for o, g in zip(out, grads) if g is not None], leaves, [g for g in grads if g is not None])
    return out, got


# ---- fe_project ------------------------------------------------------------------------------

SHAPES = [(1, 1, 1), (1, 64, 64), (3, 7, 5), (2, 1000, 33), (1, 4096, 520), (7, 129, 1024), (8, 256, 96), (9, 64, 72), (16, 320, 136),
          (17, 100, 40), (33, 72, 600), (64, 576, 264), (65, 200, 128), (129, 264, 130), (257, 192, 384), (300, 513, 257), (600, 88, 1000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_project(fe, handles, dtype, M, K, N):
    g = gen(M * 1000 + K + N)
    x, w = normal(g, dtype, M, K), normal(g, dtype, N, K, std=K ** -0.5)
    b, r, do = normal(g, dtype, N), normal(g, dtype, M, N), normal(g, dtype, M, N)
    for i, act in enumerate(("none", "relu", "silu", "gelu")):
        bias, res = (b if (i + M) % 2 else None), (r if (i + N) % 3 else None)
        want = ref.project(dict(act=act, unit=ref.UNIT[dtype]), x, w, bias, res, do)
        leaves = [v for v in (x, w, bias, res) if v is not None]

        def call(x, w, *rest):
            rest = list(rest)
            bb = rest.pop(0) if bias is not None else None
            return fe.fe_project(handles[dtype], x, w, bias=bb, act=act, residual=rest[0] if rest else None)
        (out,), got = both(call, leaves, [do])
        ref.check(out, want["out"], f"out {act}")
        ref.check(got[0], want["dx"], f"dx {act}")
        ref.check(got[1], want["dw"], f"dw {act}")
        if bias is not None:
            ref.check(got[2], want["dbias"], f"dbias {act}")
        if res is not None:
            assert torch.equal(got[-1], do)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(1, 200, 72), (5, 64, 120), (40, 136, 200), (130, 96, 264), (300, 256, 512)])
@pytest.mark.parametrize("left,right", [(0, 8), (1, 0), (3, 2), (8, 8)])
def test_project_strides(fe, handles, dtype, M, K, N, left, right):
    """Operands and outputs that are columns of wider matrices, on and off 16-byte boundaries: nothing
    around the outputs is written, and what lies around the operands does not matter."""
    t, g = handles[dtype], gen(M + K + left)
    x, w = inside(normal(g, dtype, M, K), left, right)[0], inside(normal(g, dtype, N, K, std=K ** -0.5), left, right)[0]
    r, do = inside(normal(g, dtype, M, N), left, right)[0], inside(normal(g, dtype, M, N), left, right)[0]
    want = ref.project(dict(act="silu", unit=ref.UNIT[dtype]), x, w, None, r, do)
    out, wide = inside(torch.zeros_like(r), left, right)
    pre, wide_pre = inside(torch.zeros(M, N, device="cuda"), left, right)
    assert fe.fe_project(t, x, w, act="silu", residual=r, out=out, pre=pre) is out
    ref.check(out, want["out"], "out")
    untouched(wide, left, N)
    untouched(wide_pre, left, N)
    dx, dw, db = fe.fe_project_backward(t, do, x, w, pre, "silu", dbias=True)
    for name, v in (("dx", dx), ("dw", dw), ("dbias", db)):
        ref.check(v, want[name], name)
    same = r.clone()  # in place: the residual becomes the result
    fe.fe_project(t, x, w, act="silu", residual=same, out=same)
    assert torch.equal(same, out)


def test_project_repeated_rows_and_leading_dimensions(fe, handles):
    t, g = handles["bf16"], gen(5)
    x, w = normal(g, "bf16", 64)[None].expand(6, 64), normal(g, "bf16", 40, 64)
    a, b = fe.fe_project(t, x, w), fe.fe_project(t, x.contiguous(), w)
    assert torch.equal(a, b)
    y = fe.fe_project(t, normal(g, "bf16", 2, 3, 64), w)
    assert y.shape == (2, 3, 40)
    do = normal(g, "bf16", 1)[None].expand(6, 40)  # a gradient with no strides
    _, (dx, dw) = both(lambda x, w: fe.fe_project(t, x, w), [x.contiguous(), w], [do])
    _, (ex, ew) = both(lambda x, w: fe.fe_project(t, x, w), [x.contiguous(), w], [do.contiguous()])
    assert torch.equal(dx, ex) and torch.equal(dw, ew)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows(fe, handles, dtype):
    t, g = handles[dtype], gen(1)
    x, w, b = normal(g, dtype, 0, 16), normal(g, dtype, 8, 16), normal(g, dtype, 8)
    (out,), (dx, dw, db) = both(lambda x, w, b: fe.fe_project(t, x, w, b, "silu"), [x, w, b], [normal(g, dtype, 0, 8)])
    assert out.shape == (0, 8) and dx.shape == (0, 16) and not dw.any() and not db.any()
    (out,), (dx, dg, du) = both(lambda x, g, u: fe.fe_gated_ffn(t, x, g, u), [x, w, w.clone()], [normal(g, dtype, 0, 8)])
    assert out.shape == (0, 8) and not dg.any() and not du.any()
    (y, n), (dx, dz, dw) = both(lambda x, z, w: fe.fe_block_norm(t, x, z, post_weight=w), [x, x.clone(), w[0].clone()], [x, x])
    assert y.shape == n.shape == (0, 16) and not dw.any()
    lp, ent, lse, ids, tops = fe.fe_token_logprobs(t, x, torch.zeros(0, 2, dtype=torch.int32, device="cuda"), top=3)
    assert lp.shape == (0, 2) and ids.shape == (0, 3) and ent.shape == lse.shape == (0,)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("M", [1, 40, 300])
def test_project_extremes(fe, handles, dtype, act, M):
    """Products that overflow, vanish or are not numbers, one row each: the others do not notice."""
    t, g = handles[dtype], gen(9)
    x, w = normal(g, dtype, M, 72), normal(g, dtype, 80, 72)
    i = M // 2
    for v in (math.inf, -math.inf, math.nan, 1e30, -1e30, 0.0, 1e-30):
        x[i] = 0.0
        x[i, 3] = v
        out = fe.fe_project(t, x, w, act=act)
        pre = fe.fe_project(t, x, w)
        rest = [j for j in range(M) if j != i]
        want = ref.project(dict(act=act, unit=ref.UNIT[dtype]), x[rest], w, None, None)["out"]
        ref.check(out[rest], want, "other rows")
        z = v * w[:, 3].double()
        assert torch.equal(torch.isnan(pre[i]), torch.isnan(z)), v
        p = pre[i].double()
        a = ref.act(act, p)[0]
        if act in ("silu", "gelu"):  # minus infinity times 0; the formula's 64-bit form overflows on the way to 0 and z
            a = torch.where(p < -800, torch.where(torch.isinf(p), math.nan, 0.0), torch.where(p > 800, p, a))
        e = ref.UNIT[dtype] * a.abs() + 2.0 ** -20 * a.abs() + 1e-37
        ref.check(out[i].float(), (a.float().double(), e), f"{act} of {v}")


# ---- fe_gated_ffn -----------------------------------------------------------------------------

GATED = [(1, 1, 1), (1, 64, 64), (3, 7, 5), (1, 2048, 200), (7, 129, 40), (8, 256, 96), (9, 64, 72), (17, 100, 136), (64, 576, 264),
         (65, 200, 128), (129, 264, 130), (257, 192, 320), (300, 513, 101)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,F", GATED)
def test_gated_ffn(fe, handles, dtype, M, K, F):
    t, g = handles[dtype], gen(M + K + F)
    x, do = normal(g, dtype, M, K), normal(g, dtype, M, F)
    wg, wu = (normal(g, dtype, F, K, std=K ** -0.5) for _ in range(2))
    for act in ("silu", "gelu", "relu", "none"):
        want = ref.gated(dict(act=act, unit=ref.UNIT[dtype]), x, wg, wu, do)
        (out,), (dx, dg, du) = both(lambda x, a, b: fe.fe_gated_ffn(t, x, a, b, act=act), [x, wg, wu], [do])
        for name, v in (("out", out), ("dx", dx), ("dw_gate", dg), ("dw_up", du)):
            ref.check(v, want[name], f"{name} {act}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [1, 20, 200])
@pytest.mark.parametrize("left,right", [(0, 8), (1, 2)])
def test_gated_ffn_strides(fe, handles, dtype, M, left, right):
    t, g, K, F = handles[dtype], gen(M + left), 136, 200
    both_w = normal(g, dtype, 2 * F, K, std=K ** -0.5)  # gate and up of one fused matrix
    x, do = inside(normal(g, dtype, M, K), left, right)[0], inside(normal(g, dtype, M, F), left, right)[0]
    wg, wu = both_w[:F], inside(both_w[F:].clone(), left, right)[0]
    outs = [inside(torch.zeros(M, F, dtype=dt, device="cuda"), left, right) for dt in (x.dtype, torch.float32, torch.float32)]
    out, gp, up = (o for o, _ in outs)
    fe.fe_gated_ffn(t, x, wg, wu, out=out, gate_pre=gp, up_pre=up)
    want = ref.gated(dict(act="silu", unit=ref.UNIT[dtype]), x, wg, wu, do)
    ref.check(out, want["out"], "out")
    for _, wide in outs:
        untouched(wide, left, F)
    got = fe.fe_gated_ffn_backward(t, do, gp, up, x, wg, wu)
    for name, v in zip(("dx", "dw_gate", "dw_up"), got):
        ref.check(v, want[name], name)
    for name, v in zip(("dw_gate", "dw_up"), fe.fe_gated_ffn_backward(t, do, gp, up, x=x, dx=False)[1:3]):
        ref.check(v, want[name], name)
    ref.check(fe.fe_gated_ffn_backward(t, do, gp, up, w_gate=wg, w_up=wu, dw=False)[0], want["dx"], "dx")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,F,N", [(1, 96, 200, 96), (33, 40, 72, 136), (150, 96, 333, 50), (300, 264, 520, 192)])
def test_whole_block(fe, handles, dtype, M, K, F, N):
    """The block with its down projection and residual: its result is the two operators' one after the
    other; its gradients do not round between them."""
    t, g = handles[dtype], gen(M)
    x, r, do = normal(g, dtype, M, K), normal(g, dtype, M, N), normal(g, dtype, M, N)
    wg, wu, wd = normal(g, dtype, F, K, std=K ** -0.5), normal(g, dtype, F, K, std=K ** -0.5), normal(g, dtype, N, F, std=F ** -0.5)
    want = ref.gated(dict(act="gelu", unit=ref.UNIT[dtype]), x, wg, wu, do, wd)
    (y,), got = both(lambda x, a, b, c, r: fe.fe_gated_ffn(t, x, a, b, w_down=c, act="gelu", residual=r), [x, wg, wu, wd, r], [do])
    assert torch.equal(y, fe.fe_project(t, fe.fe_gated_ffn(t, x, wg, wu, act="gelu"), wd, residual=r))
    for name, v in zip(("dx", "dw_gate", "dw_up", "dw_down"), got):
        ref.check(v, want[name], name)
    assert torch.equal(got[4], do)
    (y,), got = both(lambda x: fe.fe_gated_ffn(t, x, wg, wu, w_down=wd, act="gelu"), [x], [do])  # frozen weights
    ref.check(got[0], want["dx"], "dx alone")
    (y,), got = both(lambda c: fe.fe_gated_ffn(t, x, wg, wu, w_down=c, act="gelu"), [wd], [do])
    ref.check(got[0], want["dw_down"], "dw_down alone")


# ---- fe_block_norm ------------------------------------------------------------------------------

WIDTHS = [(5, 1), (3, 7), (70, 64), (33, 100), (9, 256), (12, 257), (6, 1000), (40, 2048), (700, 520), (11, 5120), (4, 5121), (7, 8192),
          (3, 8200), (5, 16384), (2, 16400), (1, 33000), (2, 4100)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,d", WIDTHS)
@pytest.mark.parametrize("form", range(4))
def test_block_norm(fe, handles, dtype, R, d, form):
    t, g = handles[dtype], gen(R + d + form)
    post, rows, scale, offset = [(True, R, 0.5, 0.0), (False, 0, 1.0, 1.0), (True, 1, 2.5, 1.0), (True, max(1, R // 3), -1.0, 0.0)][form]
    x, z = normal(g, dtype, R, d, std=2.0), normal(g, dtype, R, d, std=0.5)
    dy, dn = normal(g, dtype, R, d), normal(g, dtype, R, d)
    pw = normal(g, dtype, d, std=0.3) if post else None
    qw = normal(g, dtype, d, std=0.3) if form != 3 else None
    gate = normal(g, dtype, -(-R // rows), d) if rows else None
    c = dict(post=post, rows=rows, scale=scale, offset=offset, eps=1e-5, unit=ref.UNIT[dtype])
    want = ref.norm(c, x, z, pw, gate, qw, dy, dn)
    leaves = {k: v for k, v in dict(x=x, z=z, post_weight=pw, gate=gate, pre_weight=qw).items() if v is not None}
    out, got = both(lambda *v: fe.fe_block_norm(t, **dict(zip(leaves, v)), post=post, gate_rows=rows or None, scale=scale, offset=offset),
                    list(leaves.values()), [dy, dn])
    ref.check(out[0], want["y"], "y")
    ref.check(out[1], want["n"], "n")
    for k, v in zip(leaves, got):
        ref.check(v, want[{"x": "dx", "z": "dz", "post_weight": "dpost", "gate": "dgate", "pre_weight": "dpre"}[k]], "d" + k)
    for given in ((dy, None), (None, dn)):  # one output's gradient alone
        want = ref.norm(c, x, z, pw, gate, qw, *given)
        got = fe.fe_block_norm_backward(t, x, z, post, pw, gate, rows or None, scale, qw, offset, dy=given[0], dn=given[1])
        for name, v in zip(("dx", "dz", "dpost", "dgate", "dpre"), got):
            if v is not None and name in want:
                ref.check(v, want[name], f"{name} of one")
            elif v is not None:
                assert name == "dpre" and not v.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,d,rows", [(1000, 96, 1), (1000, 96, 7), (900, 1024, 2), (3000, 16, 1500), (400, 17000, 3), (400, 17000, 390),
                                      (1001, 1024, 500), (1201, 5120, 600), (701, 96, 700), (801, 8000, 400), (500, 2000, 1)])
def test_gate_groups(fe, handles, dtype, R, d, rows):
    """From a gate for each row to one for nearly all, more and fewer groups than the GPU has SMs, and a
    last group that is short."""
    t, g = handles[dtype], gen(R + rows)
    x, z, dy, dn = (normal(g, dtype, R, d) for _ in range(4))
    gate, pw = normal(g, dtype, -(-R // rows), d), normal(g, dtype, d)
    want = ref.norm(dict(post=True, rows=rows, scale=1.0, offset=0.0, eps=1e-5, unit=ref.UNIT[dtype]), x, z, pw, gate, None, dy, dn)
    got = fe.fe_block_norm_backward(t, x, z, None, pw, gate, rows, dy=dy, dn=dn)
    for name, v in zip(("dx", "dz", "dpost", "dgate"), got):
        ref.check(v, want[name], name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [132, 300, 512, 1021, 1284, 1536, 2104, 2560, 2880, 2976, 4092, 5112, 6140, 8184, 12280, 12296, 16377])
@pytest.mark.parametrize("rows", [None, 1, 3])
def test_block_norm_forms(fe, handles, dtype, d, rows):
    """Both edges of every form in which a row is held, with several rows for each worker."""
    t, g = handles[dtype], gen(d)
    R = 1 + min(3000, (1 << 22) // d)
    x, z, dy, dn = (normal(g, dtype, R, d) for _ in range(4))
    gate, pw, qw = normal(g, dtype, -(-R // rows), d) if rows else None, normal(g, dtype, d), normal(g, dtype, d)
    want = ref.norm(dict(post=True, rows=rows or 0, scale=0.5, offset=1.0, eps=1e-5, unit=ref.UNIT[dtype]), x, z, pw, gate, qw, dy, dn)
    y, n = fe.fe_block_norm(t, x, z, None, pw, gate, rows, 0.5, qw, 1.0)
    ref.check(y, want["y"], "y")
    ref.check(n, want["n"], "n")
    got = fe.fe_block_norm_backward(t, x, z, None, pw, gate, rows, 0.5, qw, 1.0, dy=dy, dn=dn)
    for name, v in zip(("dx", "dz", "dpost", "dgate", "dpre"), got):
        if v is not None:
            ref.check(v, want[name], name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [72, 1000, 9000, 20000])
@pytest.mark.parametrize("left,right", [(8, 0), (1, 2)])
def test_block_norm_strides_and_in_place(fe, handles, dtype, d, left, right):
    t, g, R = handles[dtype], gen(d), 20
    x, z, dy, dn = (inside(normal(g, dtype, R, d), left, right)[0] for _ in range(4))
    pw, qw, gate = normal(g, dtype, d), normal(g, dtype, d), inside(normal(g, dtype, 4, d), left, right)[0]
    kw = dict(post_weight=pw, gate=gate, gate_rows=5, pre_weight=qw)
    want = ref.norm(dict(post=True, rows=5, scale=1.0, offset=0.0, eps=1e-5, unit=ref.UNIT[dtype]), x, z, pw, gate, qw, dy, dn)
    outs = [inside(torch.zeros(R, d, dtype=x.dtype, device="cuda"), left, right) for _ in range(2)]
    y, n = fe.fe_block_norm(t, x, z, y=outs[0][0], n=outs[1][0], **kw)
    ref.check(y, want["y"], "y")
    ref.check(n, want["n"], "n")
    for _, wide in outs:
        untouched(wide, left, d)
    x2, z2 = inside(x.clone(), left, right)[0], inside(z.clone(), left, right)[0]
    fe.fe_block_norm(t, x2, z2, y=x2, n=z2, **kw)  # the residual stream and the block's output in place
    assert torch.equal(x2, y) and torch.equal(z2, n)
    z3 = inside(z.clone(), left, right)[0]
    fe.fe_block_norm(t, x, z3, y=z3, n=n, **kw)
    assert torch.equal(z3, y)
    got = fe.fe_block_norm_backward(t, x, z, None, pw, gate, 5, pre_weight=qw, dy=dy, dn=dn)
    for name, v in zip(("dx", "dz", "dpost", "dgate", "dpre"), got):
        ref.check(v, want[name], name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,d", [(50, 64), (50, 1000), (40, 5120), (30, 8000), (20, 20000)])
def test_block_norm_gradients_in_place(fe, handles, dtype, R, d):
    """dx and dz in the place of dy and dn, either way round."""
    t, g = handles[dtype], gen(d)
    x, z, dy, dn = (normal(g, dtype, R, d) for _ in range(4))
    pw, qw = normal(g, dtype, d), normal(g, dtype, d)
    want = fe.fe_block_norm_backward(t, x, z, None, pw, pre_weight=qw, dy=dy, dn=dn)
    from paper_2509_20416_gb300 import layer
    for swap in (False, True):
        a, b = dy.clone(), dn.clone()
        dx, dz = (b, a) if swap else (a, b)
        dp, dq = torch.empty_like(pw), torch.empty_like(qw)
        m = lambda v: (v.data_ptr(), d)
        args = layer._norm_args(t, (True, 0, 1.0, 0.0, 1e-5), x, z, pw, None, qw) + (*m(a), *m(b), *m(dx), *m(dz), 0, 0, dp.data_ptr(), dq.data_ptr())
        layer._call("fe_block_norm_backward", t, None, (x, z, pw, qw, a, b, dp, dq), args)
        for got, w in zip((dx, dz, dp, dq), (want[0], want[1], want[2], want[4])):
            assert torch.equal(got, w)


def test_norm_alone(fe, handles):
    """Without a block's output: the first norm of a model."""
    t, g = handles["bf16"], gen(2)
    x, w, dn = normal(g, "bf16", 30, 512), normal(g, "bf16", 512), normal(g, "bf16", 30, 512)
    want = ref.norm(dict(post=False, rows=0, scale=1.0, offset=0.0, eps=1e-5, unit=2.0 ** -8), x, None, None, None, w, None, dn)
    (y, n), (dx, dw) = both(lambda x, w: fe.fe_block_norm(t, x, pre_weight=w), [x, w], [None, dn])
    assert torch.equal(y, x)
    assert fe.fe_block_norm(t, x, pre_weight=w)[0] is x  # nothing is written
    copy = torch.empty_like(x)
    assert torch.equal(fe.fe_block_norm(t, x, pre_weight=w, y=copy)[1], n) and torch.equal(copy, x)
    leaf = x.detach().requires_grad_()  # the residual's gradient joins the norm's
    y, n2 = fe.fe_block_norm(t, leaf, pre_weight=w)
    d, = torch.autograd.grad([y * 1.0, n2], [leaf], [torch.ones_like(x), dn])
    assert torch.equal(d, (dx.float() + 1.0).bfloat16())
    ref.check(n, want["n"], "n")
    ref.check(dx, want["dx"], "dx")
    ref.check(dw, want["dpre"], "dw")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,d", [(20, 100), (9, 5120), (3, 20000)])
def test_norm_behind_a_block_alone(fe, handles, dtype, R, d):
    """The last block of a model: its norm, gate and residual, and no block behind it."""
    t, g = handles[dtype], gen(d)
    x, z, dy, pw, gate = (normal(g, dtype, *s) for s in ((R, d), (R, d), (R, d), (d,), (d,)))
    want = ref.norm(dict(post=True, rows=R, scale=0.5, offset=1.0, eps=1e-5, unit=ref.UNIT[dtype]), x, z, pw, gate[None], None, dy, None)

    def call(x, z, pw, gate):
        y, n = fe.fe_block_norm(t, x, z, post_weight=pw, gate=gate, scale=0.5, offset=1.0, pre=False)
        assert n is None
        return y
    (y,), got = both(call, [x, z, pw, gate], [dy])
    ref.check(y, want["y"], "y")
    for name, v in zip(("dx", "dz", "dpost"), got):
        ref.check(v, want[name], name)
    ref.check(got[3][None], want["dgate"], "dgate")
    with pytest.raises(ValueError, match="pre_weight"):
        fe.fe_block_norm(t, x, z, pre_weight=pw, pre=False)


# ---- fe_token_logprobs ------------------------------------------------------------------------------


def given(g, R, V, J, K, masked=0.0):
    tok = torch.randint(0, V, (R, J), generator=g, device="cuda", dtype=torch.int32)
    tok[torch.rand(R, J, generator=g, device="cuda") < 0.2] = -1
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    return tok, (n(R, J), n(R), n(R), n(R, K))


def check_logprobs(fe, t, x, tok, T, K, grads):
    dtype = "f32" if x.dtype == torch.float32 else "bf16"
    dl, dh, dz, dt = grads
    want = ref.logprobs(x, tok, T, K, dl, dh, dz, dt if K else None, unit=ref.UNIT[dtype], grad=True)
    leaf = x.detach().requires_grad_()
    lp, ent, lse, ids, tops = fe.fe_token_logprobs(t, leaf, tok, top=K, temperature=T)
    ref.check(lp, want["logprob"], "logprob")
    ref.check(ent, want["entropy"], "entropy")
    ref.check(lse, want["lse"], "lse")
    if K:
        assert torch.equal(ids, want["top_id"])
        ref.check(tops, want["top_logprob"], "top_logprob")
    outs, gs = [lp, ent, lse] + ([tops] if K else []), [dl, dh, dz] + ([dt] if K else [])
    d, = torch.autograd.grad(outs, [leaf], gs)
    ref.check(d, want["dlogits"], "dlogits")
    return want


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,V,J,K", [(1, 1, 1, 1), (3, 2, 2, 1), (5, 7, 3, 7), (40, 33, 1, 32), (700, 1000, 8, 5), (2, 4099, 64, 20), (33, 5000, 1, 0),
                                     (1, 128256, 2, 8), (3, 128257, 5, 32), (70, 32000, 1, 10), (1, 40001, 3, 32), (1300, 300, 2, 12),
                                     (9, 16384, 4, 3), (5, 8191, 1, 32), (2, 1 << 20, 3, 16)])
def test_token_logprobs(fe, handles, dtype, R, V, J, K):
    g = gen(R + V)
    x = normal(g, dtype, R, V, std=3.0)
    tok, grads = given(g, R, V, J, K)
    check_logprobs(fe, handles["f32"], x, tok, [1.0, 0.7, 1.9][V % 3], K, grads)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("left,right", [(0, 3), (1, 2), (5, 0), (8, 8)])
def test_token_logprobs_strides(fe, handles, dtype, left, right):
    t, g, R, V = handles["bf16"], gen(left), 6, 4100
    x, _ = inside(normal(g, dtype, R, V, std=3.0), left, right)
    tok, grads = given(g, R, V, 3, 9)
    want = check_logprobs(fe, t, x, tok, 1.0, 9, grads)
    stats = torch.empty(R, 2, device="cuda")
    lp, ent, lse, ids, tops = fe.fe_token_logprobs(t, x, tok, top=9, stats=stats)
    d, wide = inside(torch.zeros_like(x), (left + 1) % 8, right)  # (another alignment than the logits')
    fe.fe_token_logprobs_backward(t, x, stats, tok, grads[0], ent, grads[1], grads[2], ids, grads[3], dlogits=d)
    ref.check(d, want["dlogits"], "dlogits")
    untouched(wide, (left + 1) % 8, V)
    fe.fe_token_logprobs_backward(t, x, stats, tok, grads[0], ent, grads[1], grads[2], ids, grads[3], dlogits=x)  # in place
    assert torch.equal(x, d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [50, 5003, 130000])
def test_token_logprobs_masks_and_ties(fe, handles, dtype, V):
    """Ruled-out tokens, rows without any token, the type's lowest value, equal logits, infinities and NaN."""
    g, K, J = gen(V), 6, 3
    x = normal(g, dtype, 12, V, std=2.0)
    x[0, torch.rand(V, generator=g, device="cuda") < 0.5] = -math.inf
    x[1] = -math.inf
    x[2] = -math.inf
    x[2, V // 2] = 0.25  # one token left
    x[3] = torch.finfo(x.dtype).min
    x[4] = torch.finfo(x.dtype).min
    x[4, 3:9] = 1.0
    x[5] = 1.5  # all equal
    x[6] = (x[6] * 2).round() / 2  # many equal
    x[7, V - 2] = math.nan
    x[8, 5] = math.inf
    x[9] = torch.arange(V, device="cuda", dtype=torch.float32).to(x.dtype) / V  # growing: runs of equal ones in bfloat16
    x[10] = -x[9]
    x[11, :] = 0.0
    x[11, ::2] = -0.0
    tok, grads = given(g, 12, V, J, K)
    tok[1, 0], tok[2, 0], tok[2, 1], tok[7, 0], tok[8, 0] = 3, V // 2, 0, 1, 5
    tok[0, :] = tok[0, 0]  # the same token again
    for T in (1.0, 0.5):
        dl, dh, dz, dt = (v.clone() for v in grads)
        check_logprobs(fe, handles["f32"], x, tok, T, K, (dl, dh, dz, dt))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,stride", [(65536, 512 * 8), (65536, 4096), (131072, 1), (131072, 2048), (200000, 4)])
def test_largest_logits_in_one_place(fe, handles, dtype, V, stride):
    """The largest elements all fall to one thread, or to neighbouring ones, with equal values behind them."""
    g = gen(V)
    x = normal(g, dtype, 2, V).clamp(-4, 4)
    at = torch.arange(3, V, stride, device="cuda")[:2000]
    x[0, at] = 8.0 + torch.randint(0, 3, at.shape, generator=g, device="cuda").to(x.dtype)
    x[1, at] = 8.0
    tok, grads = given(g, 2, V, 1, 32)
    check_logprobs(fe, handles["f32"], x, tok, 1.0, 32, grads)


def test_tokens_out_of_range(fe, handles):
    t, g = handles["f32"], gen(4)
    x = normal(g, "f32", 3, 100)
    tok = torch.tensor([[1, 100], [5, 6], [2147483647, 7]], dtype=torch.int32, device="cuda")
    stats = torch.empty(3, 2, device="cuda")
    lp, ent, lse, *_ = fe.fe_token_logprobs(t, x, tok, stats=stats)
    assert fe.fe_target_status(t) == fe.FE_ERR_DEVICE
    assert lp[0, 1] == 0 and lp[2, 0] == 0
    d = fe.fe_token_logprobs_backward(t, x, stats, tok, torch.ones(3, 2, device="cuda"))
    assert fe.fe_target_status(t) == fe.FE_ERR_DEVICE
    want = ref.logprobs(x, tok, 1.0, 0, torch.ones(3, 2, device="cuda"), grad=True)
    ref.check(lp, want["logprob"], "logprob")
    ref.check(d, want["dlogits"], "dlogits")


# ---- calls as programs make them ------------------------------------------------------------------


def steps(fe, t, dtype, seed=0, M=37):
    """A layer's dense part and its answer, with the gradients of everything; returns all results."""
    g = gen(seed)
    d, F, V = 136, 264, 1003
    n = lambda *s, std=1.0: normal(g, dtype, *s, std=std).requires_grad_()
    x, wo, pw, qw, gate = n(M, d), n(d, d, std=d ** -0.5), n(d), n(d), n(d)
    wg, wu, wd, head, bias = n(F, d, std=d ** -0.5), n(F, d, std=d ** -0.5), n(d, F, std=F ** -0.5), n(V, d, std=d ** -0.5), n(V)
    tok = torch.randint(-1, V, (M, 2), generator=g, device="cuda", dtype=torch.int32)
    dl, dh = torch.randn(M, 2, generator=g, device="cuda"), torch.randn(M, generator=g, device="cuda")
    leaves = [x, wo, pw, qw, gate, wg, wu, wd, head, bias]

    def run():
        o = fe.fe_project(t, x, wo, act="gelu")
        y, u = fe.fe_block_norm(t, x, o, post_weight=pw, gate=gate, scale=0.5, pre_weight=qw)
        f = fe.fe_gated_ffn(t, u, wg, wu, w_down=wd, residual=y)
        _, u = fe.fe_block_norm(t, f, pre_weight=qw)
        logits = fe.fe_project(t, u, head, bias=bias)
        lp, ent, lse, ids, tops = fe.fe_token_logprobs(t, logits, tok, top=4)
        return [logits, lp, ent, ids, tops, *torch.autograd.grad([lp, ent], leaves, [dl, dh])]
    return run, leaves


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [1, 37, 300])
def test_layer_in_one_go(fe, handles, dtype, M):
    """The operators one after another, against the same chain in float64 autograd: every result within a
    share of its norm that the chain's roundings explain (some ten of them, each UNIT of what it rounds)."""
    t = handles[dtype]
    run, leaves = steps(fe, t, dtype, M, M)
    got = run()
    again = run()
    assert all(torch.equal(a, b) for a, b in zip(got, again))  # (no order depends on timing)
    x, wo, pw, qw, gate, wg, wu, wd, head, bias = v = [p.detach().double().requires_grad_() for p in leaves]
    norm = lambda a, w: a * (a.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w
    o = torch.nn.functional.gelu(x @ wo.T, approximate="tanh")
    y = x + 0.5 * gate * norm(o, pw)
    u = norm(y, qw)
    f = y + (torch.nn.functional.silu(u @ wg.T) * (u @ wu.T)) @ wd.T
    logits = norm(f, qw) @ head.T + bias
    g = gen(M)  # (the inputs again, up to the tokens)
    d, F, V = 136, 264, 1003
    for s in ((M, d), (d, d), (d,), (d,), (d,), (F, d), (F, d), (d, F), (V, d), (V,)):
        torch.randn(s, generator=g, device="cuda")
    tok = torch.randint(-1, V, (M, 2), generator=g, device="cuda", dtype=torch.int32).long()
    dl, dh = torch.randn(M, 2, generator=g, device="cuda"), torch.randn(M, generator=g, device="cuda")
    logp = torch.log_softmax(logits, 1)
    lp = torch.where(tok >= 0, logp.gather(1, tok.clamp(min=0)), 0.0)
    ent = -(logp.exp() * logp).sum(1)
    want = [logits, lp, ent, None, None, *torch.autograd.grad([lp, ent], v, [dl.double(), dh.double()])]
    share = 12 * ref.UNIT[dtype] if dtype == "bf16" else 2.0 ** -14
    for i, (a, b) in enumerate(zip(got, want)):
        if b is not None:
            assert (a.double() - b).norm() <= share * b.norm() + 1e-9, i


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_step(fe, handles, dtype):
    """A whole step, backward pass included, captured in a graph and replayed with new inputs; a second graph
    of the same handle replays next to it."""
    t = handles[dtype]
    run, leaves = steps(fe, t, dtype, 3)
    want = [r.detach().clone() for r in run()]
    other, _ = steps(fe, t, dtype, 4)
    want_other = [r.detach().clone() for r in other()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
        other()
    torch.cuda.current_stream().wait_stream(s)
    graphs, results = [], []
    for f in (run, other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = f()
        graphs.append(graph)
        results.append(out)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(a):
            graphs[0].replay()
        with torch.cuda.stream(b):
            graphs[1].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(results[0], want))
    assert all(torch.equal(x, y) for x, y in zip(results[1], want_other))
    with torch.no_grad():
        leaves[0].mul_(0.5)
    graphs[0].replay()
    assert all(torch.equal(x, y) for x, y in zip(results[0], run()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_gradients_beside_a_living_graph(fe, handles, dtype):
    """Gradients by plain calls are captured while an eager graph of the same leaves lives, and that graph's
    own backward pass gives the same afterwards."""
    t, g = handles[dtype], gen(12)
    x, wg, wu, wd = normal(g, dtype, 150, 96), normal(g, dtype, 200, 96), normal(g, dtype, 200, 96), normal(g, dtype, 96, 200)
    do = normal(g, dtype, 150, 96)
    leaves = [v.detach().requires_grad_() for v in (x, wg, wu, wd)]
    alive = fe.fe_gated_ffn(t, *leaves)

    def step():
        gp, up = torch.empty(150, 200, device="cuda"), torch.empty(150, 200, device="cuda")
        fe.fe_gated_ffn(t, x, wg, wu, wd, gate_pre=gp, up_pre=up)
        return fe.fe_gated_ffn_backward(t, do, gp, up, x, wg, wu, wd)
    want = step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for v in got:
        v.zero_()
    graph.replay()
    eager = torch.autograd.grad([alive], leaves, [do])
    for a, b, c in zip(got, want, eager):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_other_streams(fe, handles, dtype):
    """Calls on a stream of their own run there, behind what is queued on it: inputs that the stream makes
    late are seen."""
    t, g = handles[dtype], gen(8)
    x, w, r = normal(g, dtype, 40, 64), normal(g, dtype, 72, 64), normal(g, dtype, 40, 72)
    pw = normal(g, dtype, 72)
    tok = torch.zeros(40, 1, dtype=torch.int32, device="cuda")
    want = fe.fe_project(t, x, w, act="silu", residual=r)
    norm = fe.fe_block_norm(t, r, want, post_weight=pw)
    logp = fe.fe_token_logprobs(t, norm[1], tok, top=3)
    dx, dw, db = fe.fe_project_backward(t, norm[1], x, w, dbias=True)
    s = torch.cuda.Stream()
    late = torch.zeros_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(50_000_000)
        late.copy_(x)
    y = fe.fe_project(t, late, w, act="silu", residual=r, stream=s)
    z = fe.fe_block_norm(t, r, y, post_weight=pw, stream=s)
    lp = fe.fe_token_logprobs(t, z[1], tok, top=3, stream=s.cuda_stream)
    got = fe.fe_project_backward(t, z[1], late, w, dbias=True, stream=s)
    wide = torch.zeros(40, 2, dtype=torch.int32, device="cuda")  # tokens that are not contiguous, and made late
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(50_000_000)
        wide[:, 0] = 5
    late_lp = fe.fe_token_logprobs(t, z[1], wide[:, :1], stream=s)[0]
    s.synchronize()
    assert torch.equal(late_lp, fe.fe_token_logprobs(t, z[1], wide[:, :1].contiguous())[0])
    for a, b in zip((y, *z, *lp, *got), (want, *norm, *logp, dx, dw, db)):
        assert torch.equal(a, b)


def test_gradients_against_differences(fe, handles):
    """The float32 operators' gradients against differences of their own results along random directions: a
    central difference with step h is off by h^2 / 6 of a third derivative and by roundings of the sum that
    is differenced, 2^-20 of its terms over h."""
    t, h = handles["f32"], 2.0 ** -6
    run, leaves = steps(fe, t, "f32", 5)
    got = run()[5:]
    g = gen(50)
    for i, p in enumerate(leaves):
        v = torch.randn(p.shape, generator=g, device="cuda")
        v = v / v.norm()
        base = p.detach().clone()
        ends = []
        for sign in (1, -1):
            with torch.no_grad():
                p.copy_(base + sign * h * v)
            o = run()
            gg = gen(5)
            M, d, F, V = 37, 136, 264, 1003
            for s in ((M, d), (d, d), (d,), (d,), (d,), (F, d), (F, d), (d, F), (V, d), (V,)):
                torch.randn(s, generator=gg, device="cuda")
            torch.randint(-1, V, (M, 2), generator=gg, device="cuda", dtype=torch.int32)
            dl, dh = torch.randn(M, 2, generator=gg, device="cuda"), torch.randn(M, generator=gg, device="cuda")
            terms = torch.cat([(o[1] * dl).flatten(), o[2] * dh]).double()
            ends.append((terms.sum(), terms.abs().sum()))
        with torch.no_grad():
            p.copy_(base)
        have = (got[i].double() * v).sum()
        want = (ends[0][0] - ends[1][0]) / (2 * h)
        size = got[i].double().norm()
        assert abs(have - want) <= 2.0 ** -20 * ends[0][1] / h + h * h * 40 * (1 + size), (i, float(have), float(want))


def test_offsets_past_32_bits(fe, handles):
    """Logits of more than 2^31 elements, from a matrix product: rows at both ends."""
    t, g, R, V = handles["bf16"], gen(6), 17000, 128264
    x, w = normal(g, "bf16", R, 64), normal(g, "bf16", V, 64, std=0.125)
    logits = fe.fe_project(t, x, w)
    assert logits.numel() > 1 << 31
    tok = torch.randint(0, V, (R, 1), generator=g, device="cuda", dtype=torch.int32)
    stats = torch.empty(R, 2, device="cuda")
    lp, ent, lse, ids, tops = fe.fe_token_logprobs(t, logits, tok, top=3, stats=stats)
    rows = torch.tensor([0, 1, 8000, R - 2, R - 1], device="cuda")
    want = ref.project(dict(act="none", unit=2.0 ** -8), x[rows], w, None, None)["out"]
    ref.check(logits[rows], want, "logits")
    dl, dh = torch.randn(R, 1, generator=g, device="cuda"), torch.randn(R, generator=g, device="cuda")
    want = ref.logprobs(logits[rows], tok[rows], 1.0, 3, dl[rows], dh[rows], unit=2.0 ** -8, grad=True)
    ref.check(lp[rows], want["logprob"], "logprob")
    assert torch.equal(ids[rows], want["top_id"])
    d = fe.fe_token_logprobs_backward(t, logits, stats, tok, dl, ent, dh)
    ref.check(d[rows], want["dlogits"], "dlogits")
    dx, dw, db = fe.fe_project_backward(t, d, x, w, dbias=True)
    q = ref.Product(d[rows], w.double().T)
    ref.check(dx[rows], (q.v, q.err + 2.0 ** -8 * (q.v.abs() + q.err)), "dx")
    at = torch.tensor([0, 5, V - 1], device="cuda")
    q = ref.Product(d[:, at].T, x.T)
    ref.check(dw[at], (q.v, q.err + 2.0 ** -8 * (q.v.abs() + q.err)), "dw")


def test_binding_refuses(fe, handles):
    t, g = handles["bf16"], gen(1)
    x, w = normal(g, "bf16", 4, 16), normal(g, "bf16", 8, 16)
    bad = [lambda: fe.fe_project(t, x.float(), w), lambda: fe.fe_project(t, x[:, :8], w), lambda: fe.fe_project(t, x, w, bias=w[:, 0]),
           lambda: fe.fe_project(t, x.T, w[:, :4]), lambda: fe.fe_project(t, x, w, residual=x), lambda: fe.fe_project(t, x, w, act="tanh"),
           lambda: fe.fe_gated_ffn(t, x, w, w[:4]), lambda: fe.fe_block_norm(t, x, x[:2]), lambda: fe.fe_block_norm(t, x, x, gate=x, gate_rows=2),
           lambda: fe.fe_token_logprobs(t, x, torch.zeros(4, 1, dtype=torch.int64, device="cuda")),
           lambda: fe.fe_token_logprobs(t, x.double()), lambda: fe.fe_token_logprobs(t, x, torch.zeros(3, 1, dtype=torch.int32, device="cuda"))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: fe.fe_token_logprobs(t, x, top=17), lambda: fe.fe_token_logprobs(t, x, temperature=0.0),
                 lambda: fe.fe_block_norm(t, x, eps=-1.0), lambda: fe.fe_block_norm(t, x, x, scale=math.inf)):
        with pytest.raises(fe.FeError) as e:
            call()
        assert e.value.code == fe.FE_ERR_INVALID_ARG
    y = fe.fe_project(t, x.requires_grad_(), w)
    with pytest.raises(RuntimeError):  # differentiable once
        d, = torch.autograd.grad(y.float().square().sum(), [x], create_graph=True)
        d.sum().backward()
