"""The matrix products in the modes of large calls (gemm_shapes.py), every result against 64 bits: several tiles a
pair of CTAs, so that both accumulators, the waits between a tile's end and the next, and slots of the rings
are used again; each form at each width; large float32 tiles; rings of few rows that turn."""
import pytest
import torch

import gemm_shapes as shapes
import layer_ref as ref
from test_gpu_layer import both, fe, gen, handles, no_status, normal  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,size", [("bf16", s) for s in shapes.BLOCKS + shapes.ODD_BLOCKS] +
                         [("f32", s) for s in shapes.BLOCKS[2:6] + shapes.ODD_BLOCKS], ids=str)
def test_blocks(fe, handles, dtype, size):  # noqa: F811
    (M, K, F, N), t = size, handles[dtype]
    g = gen(M + K)
    x, r, do = normal(g, dtype, M, K), normal(g, dtype, M, N), normal(g, dtype, M, N)
    wg, wu, wd = normal(g, dtype, F, K, std=K ** -0.5), normal(g, dtype, F, K, std=K ** -0.5), normal(g, dtype, N, F, std=F ** -0.5)
    c = dict(act="silu", unit=ref.UNIT[dtype])
    gp, up = torch.empty(M, F, device="cuda"), torch.empty(M, F, device="cuda")
    h = fe.fe_gated_ffn(t, x, wg, wu, gate_pre=gp, up_pre=up)
    want = ref.gated(c, x, wg, wu, do, wd)
    ref.check(h, want["out"], "h")
    for name, pre, w in (("gate", gp, wg), ("up", up, wu)):
        p = ref.Product(x, w)
        ref.check(pre, (p.v, p.err), name)
    y = fe.fe_project(t, h, wd, residual=r)
    ref.check(y, ref.project(dict(act="none", unit=c["unit"]), h, wd, None, r)["out"], "y")
    got = fe.fe_gated_ffn_backward(t, do, gp, up, x, wg, wu, wd)
    for name, v in zip(("dx", "dw_gate", "dw_up", "dw_down"), got):
        ref.check(v, want[name], name)
    again = fe.fe_gated_ffn_backward(t, do, gp, up, x, wg, wu, wd)
    assert all(torch.equal(a, b) for a, b in zip(got, again)) and torch.equal(h, fe.fe_gated_ffn(t, x, wg, wu))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("M,K,N", shapes.PROJECTS)
def test_projects(fe, handles, dtype, act, M, K, N):  # noqa: F811
    t, g = handles[dtype], gen(M + N)
    x, w = normal(g, dtype, M, K), normal(g, dtype, N, K, std=K ** -0.5)
    b, r, do = normal(g, dtype, N), normal(g, dtype, M, N), normal(g, dtype, M, N)
    want = ref.project(dict(act=act, unit=ref.UNIT[dtype]), x, w, b, r, do)
    pre = torch.empty(M, N, device="cuda")
    same = r.clone()
    out = fe.fe_project(t, x, w, b, act, r, pre=pre)
    ref.check(out, want["out"], "out")
    ref.check(pre, ref.project(dict(act="none", unit=0.0), x, w, b, None)["out"], "pre")
    assert torch.equal(fe.fe_project(t, x, w, b, act, same, out=same), out)
    for name, v in zip(("dx", "dw", "dbias"), fe.fe_project_backward(t, do, x, w, pre, act, dbias=True)):
        ref.check(v, want[name], name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", shapes.FEW)
def test_few_rows(fe, handles, dtype, M, K, N):  # noqa: F811
    t, g = handles[dtype], gen(M + N)
    x, w = normal(g, dtype, M, K), normal(g, dtype, N, K, std=K ** -0.5)
    b, r = normal(g, dtype, N), normal(g, dtype, M, N)
    pre = torch.empty(M, N, device="cuda")
    out = fe.fe_project(t, x, w, b, "gelu", r, pre=pre)
    ref.check(out, ref.project(dict(act="gelu", unit=ref.UNIT[dtype]), x, w, b, r)["out"], "out")
    ref.check(pre, ref.project(dict(act="none", unit=0.0), x, w, b, None)["out"], "pre")
    assert torch.equal(fe.fe_project(t, x, w, b, "gelu", r), out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,F", shapes.FEW_GATED)
def test_few_rows_gated(fe, handles, dtype, M, K, F):  # noqa: F811
    t, g = handles[dtype], gen(M + F)
    x = normal(g, dtype, M, K)
    wg, wu = normal(g, dtype, F, K, std=K ** -0.5), normal(g, dtype, F, K, std=K ** -0.5)
    gp, up = torch.empty(M, F, device="cuda"), torch.empty(M, F, device="cuda")
    out = fe.fe_gated_ffn(t, x, wg, wu, gate_pre=gp, up_pre=up)
    ref.check(out, ref.gated(dict(act="silu", unit=ref.UNIT[dtype]), x, wg, wu)["out"], "out")
    for name, pre, w in (("gate", gp, wg), ("up", up, wu)):
        p = ref.Product(x, w)
        ref.check(pre, (p.v, p.err), name)
    assert torch.equal(fe.fe_gated_ffn(t, x, wg, wu), out)
