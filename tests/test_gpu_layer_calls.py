"""Calls of the dense operators that programs may make at the edge of what include/fe_layer.h and the binding
allow."""
import os
import subprocess
import sys

import pytest
import torch

import layer_ref as ref
from test_gpu_layer import fe, gen, handles, no_status, normal  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [96, 1000, 20000])
def test_gates_of_more_rows_than_there_are(fe, handles, dtype, d):  # noqa: F811
    """One gate for all rows, by any number of rows from theirs on."""
    t, g, R = handles[dtype], gen(d), 40
    x, z, dy, dn = (normal(g, dtype, R, d) for _ in range(4))
    gate, pw = normal(g, dtype, 1, d), normal(g, dtype, d)
    want = ref.norm(dict(post=True, rows=R, scale=1.0, offset=0.0, eps=1e-5, unit=ref.UNIT[dtype]), x, z, pw, gate, None, dy, dn)
    for rows in (R, R + 1, 1 << 31, (1 << 63) - 1):
        y, n = fe.fe_block_norm(t, x, z, post_weight=pw, gate=gate, gate_rows=rows)
        ref.check(y, want["y"], "y")
        ref.check(n, want["n"], "n")
        got = fe.fe_block_norm_backward(t, x, z, None, pw, gate, rows, dy=dy, dn=dn)
        for name, v in zip(("dx", "dz", "dpost", "dgate"), got):
            ref.check(v, want[name], name)


def test_dropped_inputs_of_another_stream(fe, handles):  # noqa: F811
    """Inputs that are not contiguous are copied on the call's stream. A caller may drop them at once: memory that
    is then handed out on the current stream is not theirs while the copy waits."""
    t, g, R, V = handles["f32"], gen(3), 4096, 64
    logits = normal(g, "f32", R, V)
    tok = torch.randint(0, V, (R, 2), generator=g, device="cuda", dtype=torch.int32)
    grads = torch.randn(R, 2, generator=g, device="cuda")
    stats = torch.empty(R, 2, device="cuda")
    want = fe.fe_token_logprobs(t, logits, tok[:, :1].contiguous(), stats=stats)[0]
    want_d = fe.fe_token_logprobs_backward(t, logits, stats, tok[:, :1].contiguous(), grads[:, :1].contiguous())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    fe.fe_token_logprobs(t, logits, tok[:, :1], stream=s)  # (kernels loaded before the pause)
    torch.cuda.synchronize()
    for call in range(2):
        ids, dl = tok.clone(), grads.clone()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            torch.cuda._sleep(100_000_000)
        if call == 0:
            got = fe.fe_token_logprobs(t, logits, ids[:, :1], stream=s)[0]
        else:
            got = fe.fe_token_logprobs_backward(t, logits, stats, ids[:, :1], dl[:, :1], stream=s)
        del ids, dl
        others = [torch.full((R, 2), 7, dtype=torch.int32, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        assert torch.equal(got, want if call == 0 else want_d), call
        assert all((o == 7).all() for o in others)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(3, 900, 333), (90, 1500, 131), (300, 200, 77), (1501, 136, 4099), (2817, 72, 2050)])
def test_ragged_edges(fe, handles, dtype, M, K, N):  # noqa: F811
    """Edges at which the lanes of a warp have different numbers of columns and rows to read, in one tile and in
    several of a CTA, with all that a product's end reads and writes."""
    t, g = handles[dtype], gen(M + N)
    x, w = normal(g, dtype, M, K), normal(g, dtype, N, K, std=K ** -0.5)
    b, r = normal(g, dtype, N), normal(g, dtype, M, N)
    pre = torch.empty(M, N, device="cuda")
    c = dict(act="silu", unit=ref.UNIT[dtype])
    out = fe.fe_project(t, x, w, b, "silu", r, pre=pre)
    ref.check(out, ref.project(c, x, w, b, r)["out"], "out")
    ref.check(pre, ref.project(dict(act="none", unit=0.0), x, w, b, None)["out"], "pre")
    if N % 2:
        want = ref.logprobs(out.float(), torch.zeros(M, 1, dtype=torch.int32, device="cuda"), 1.0, 5)
        ent, lse, ids = fe.fe_token_logprobs(t, out.float(), top=5)[1:4]
        ref.check(ent, want["entropy"], "entropy")
        ref.check(lse, want["lse"], "lse")
        assert torch.equal(ids, want["top_id"])


def test_weight_gradient_of_the_most_rows(fe, handles):  # noqa: F811
    """2^30 rows, which one pair of CTAs sums in seconds: nothing gives up on it. Most rows are zeros, so that the
    few others' sum is known."""
    t, g, M, N, K = handles["bf16"], gen(30), 1 << 30, 8, 16
    dout, x = (torch.zeros(M, n, dtype=torch.bfloat16, device="cuda") for n in (N, K))
    at = torch.randint(0, M, (1000,), generator=g, device="cuda").unique()
    at = torch.cat([at, torch.tensor([M - 1], device="cuda")]).unique()
    dout[at], x[at] = normal(g, "bf16", len(at), N), normal(g, "bf16", len(at), K)
    _, dw, _ = fe.fe_project_backward(t, dout, x, dx=False)
    assert fe.fe_target_status(t) == fe.FE_OK
    q = ref.Product(dout[at].T, x[at].T)
    ref.check(dw, (q.v, q.err + 2.0 ** -8 * (q.v.abs() + q.err)), "dw")
    del dout, x
    torch.cuda.empty_cache()


def test_saved_tensors_that_are_overwritten(fe, handles):  # noqa: F811
    """A graph whose saved tensor has been taken as an output refuses to go back, as it does after PyTorch's own
    in-place operations."""
    t, g = handles["f32"], gen(11)
    x, z, w = normal(g, "f32", 12, 64), normal(g, "f32", 12, 64), normal(g, "f32", 64, 64)
    leaf = w.detach().requires_grad_()
    for write in (lambda s: fe.fe_project(t, x, w, out=s), lambda s: fe.fe_project(t, x, w, pre=s), lambda s: fe.fe_block_norm(t, x, z, y=s),
                  lambda s: fe.fe_block_norm(t, x, z, n=s), lambda s: fe.fe_gated_ffn(t, x, w, w, gate_pre=s, up_pre=torch.empty_like(s)),
                  lambda s: fe.fe_gated_ffn(t, x, w, w, w, out=s),
                  lambda s: fe.fe_token_logprobs_backward(t, x, torch.zeros(12, 2, device="cuda"), dlogits=s)):
        s = z.clone()
        for y in (s @ leaf.T, fe.fe_project(t, s, leaf)):
            write(s)
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                y.sum().backward()
        y = fe.fe_project(t, s, leaf)  # (saved as it is now)
        torch.autograd.grad([y], [leaf], [x])
    stats = torch.empty(12, 2, device="cuda")
    before = stats._version
    fe.fe_token_logprobs(t, x, stats=stats)
    assert stats._version > before


FIRST_CALLS = """
import ctypes, sys
import torch
import paper_2509_20416_gb300 as fe

class Handle(ctypes.Structure):  # the start of the library's handle
    _fields_ = [("cfg", fe.target.fe_target_config), ("device", ctypes.c_int), ("num_sms", ctypes.c_int), ("buffers", ctypes.c_void_p * 5),
                ("ready", ctypes.c_uint)]
ready = lambda: Handle.from_address(t.ptr).ready
dtype = sys.argv[1]
T = dict(f32=torch.float32, bf16=torch.bfloat16)[dtype]
t = fe.fe_target_init(dict(n_heads=2, n_kv_heads=1, head_dim=64, max_seq=16, dtype=dtype, rope_theta=1e4))
g = torch.Generator(device="cuda").manual_seed(1)
n = lambda *s: torch.randn(s, generator=g, device="cuda").to(T)
pos = torch.zeros(1, 4, dtype=torch.int32, device="cuda")
fe.fe_rope(t, n(1, 4, 2, 64), None, pos)
assert ready() == 0  # (rotating and attending need none of the dense operators' kernels)
x, w, z, v, do = n(200, 640), n(640, 640) / 25, n(200, 640), n(640), n(200, 640)
logits, tok = n(200, 33000), torch.zeros(200, 1, dtype=torch.int32, device="cuda")

def step():
    y, u = fe.fe_block_norm(t, x, z, post_weight=v, pre_weight=v)
    out = fe.fe_project(t, u, w, residual=y)
    one = fe.fe_gated_ffn(t, u[:3], w, w)
    stats = torch.empty(200, 2, device="cuda")
    lp = fe.fe_token_logprobs(t, logits, tok, top=3, stats=stats)
    back = fe.fe_token_logprobs_backward(t, logits, stats, tok, torch.ones_like(lp[0]))
    return [y, u, out, one, *lp, back, *fe.fe_project_backward(t, do, u, w, dbias=True),
            *[r for r in fe.fe_block_norm_backward(t, x, z, None, v, pre_weight=v, dy=do, dn=do) if r is not None]]

torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):  # the first calls of the process
    got = step()
assert ready() != 0
for r in got:
    r.zero_()
graph.replay()
want = step()
torch.cuda.synchronize()
assert fe.fe_target_status(t) == fe.FE_OK
for i, (a, b) in enumerate(zip(got, want)):
    assert torch.equal(a, b), i
other = fe.fe_target_init(dict(n_heads=1, n_kv_heads=1, head_dim=64, max_seq=16, dtype=dtype, rope_theta=1e4))
assert torch.equal(fe.fe_project(other, u := want[1], w, residual=want[0]), want[2])
print("first calls captured")
"""


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_first_calls_of_a_process(tmp_path, dtype):
    """A handle sets up the dense operators' kernels when they are first used, and that may be while a graph is
    captured."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    script = tmp_path / "first_calls.py"
    script.write_text(FIRST_CALLS)
    r = subprocess.run([sys.executable, str(script), dtype], cwd=root, env=dict(os.environ, PYTHONPATH=root), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "first calls captured" in r.stdout, r.stdout + r.stderr
