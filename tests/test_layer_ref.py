"""The 64-bit forms' gradients (layer_ref.py) against differences, and the layer calls' refusals and
argument layout, all without a GPU."""
import ctypes
import math
import os
import re
import struct
import subprocess

import pytest
import torch

import layer_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STEP = 2.0 ** -10


def slope(f, x, v):
    """(f(x + h v) - f(x - h v)) / 2 h, with the h^2 term taken out by a second pair."""
    d = lambda h: (f(x + h * v) - f(x - h * v)) / (2 * h)
    return (4 * d(STEP / 2) - d(STEP)) / 3


def agrees(f, x, grad, g, kinks=False):
    """grad against differences of f along random directions. Truncation leaves h^4 / 480 of a fifth
    derivative, far below 1e-8 at these sizes; rounding 2^-52 / h of f."""
    for _ in range(4):
        v = torch.randn(x.shape, generator=g, dtype=torch.float64)
        want, have = slope(f, x, v), (grad * v).sum()
        assert abs(want - have) <= 1e-8 * (1 + (grad * v).abs().sum()), (float(want), float(have))


def normal(g, *shape):
    return torch.randn(shape, generator=g, dtype=torch.float64)


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_project_gradients(act):
    g = torch.Generator().manual_seed(1)
    x, w, b, r, do = normal(g, 5, 7), normal(g, 4, 7), normal(g, 4), normal(g, 5, 4), normal(g, 5, 4)
    c = dict(act=act, unit=0.0)
    f = lambda **k: (ref.project(c, k.get("x", x), k.get("w", w), k.get("b", b), r)["out"][0] * do).sum()
    got = ref.project(c, x, w, b, r, do)
    agrees(lambda v: f(x=v), x, got["dx"][0], g)
    agrees(lambda v: f(w=v), w, got["dw"][0], g)
    agrees(lambda v: f(b=v), b, got["dbias"][0], g)


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_gated_gradients(act):
    g = torch.Generator().manual_seed(2)
    x, wg, wu, do = normal(g, 5, 7), normal(g, 6, 7), normal(g, 6, 7), normal(g, 5, 6)
    c = dict(act=act, unit=0.0)
    f = lambda **k: (ref.gated(c, k.get("x", x), k.get("wg", wg), k.get("wu", wu))["out"][0] * do).sum()
    got = ref.gated(c, x, wg, wu, do)
    agrees(lambda v: f(x=v), x, got["dx"][0], g)
    agrees(lambda v: f(wg=v), wg, got["dw_gate"][0], g)
    agrees(lambda v: f(wu=v), wu, got["dw_up"][0], g)
    wd, do = normal(g, 3, 6), normal(g, 5, 3)  # the whole block
    f = lambda **k: (ref.gated(c, k.get("x", x), wg, wu)["out"][0] @ k.get("wd", wd).T * do).sum()
    got = ref.gated(c, x, wg, wu, do, wd)
    agrees(lambda v: f(x=v), x, got["dx"][0], g)
    agrees(lambda v: f(wd=v), wd, got["dw_down"][0], g)


def test_relu_gradient_away_from_its_kink():
    z = torch.tensor([-2.0, -0.5, 0.5, 3.0], dtype=torch.float64)
    v, d = ref.act("relu", z)
    assert torch.equal(v, torch.tensor([0.0, 0.0, 0.5, 3.0], dtype=torch.float64))
    assert torch.equal(d, torch.tensor([0.0, 0.0, 1.0, 1.0], dtype=torch.float64))


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("rows", [0, 1, 2, 5])
def test_norm_gradients(post, rows):
    g = torch.Generator().manual_seed(3)
    R, d = 5, 9
    x, z, dy, dn = (normal(g, R, d) for _ in range(4))
    pw, qw = normal(g, d) if post else None, normal(g, d)
    gate = normal(g, -(-R // rows), d) if rows else None
    c = dict(post=post, rows=rows, scale=0.7, offset=0.25, eps=1e-3, unit=0.0)

    def f(**k):
        o = ref.norm(c, k.get("x", x), k.get("z", z), k.get("pw", pw), k.get("gate", gate), k.get("qw", qw))
        return (o["y"][0] * dy).sum() + (o["n"][0] * dn).sum()
    got = ref.norm(c, x, z, pw, gate, qw, dy, dn)
    agrees(lambda v: f(x=v), x, got["dx"][0], g)
    agrees(lambda v: f(z=v), z, got["dz"][0], g)
    agrees(lambda v: f(qw=v), qw, got["dpre"][0], g)
    if post:
        agrees(lambda v: f(pw=v), pw, got["dpost"][0], g)
    if rows:
        agrees(lambda v: f(gate=v), gate, got["dgate"][0], g)


def test_logprob_gradients():
    g = torch.Generator().manual_seed(4)
    R, V, J, K, T = 4, 11, 3, 2, 0.7
    x = normal(g, R, V)
    tok = torch.randint(0, V, (R, J), generator=g)
    tok[1, 1], tok[2] = -1, tok[2, 0].clone()  # none, and the same token three times
    dl, dh, dz, dt = normal(g, R, J), normal(g, R), normal(g, R), normal(g, R, K)

    def f(v):
        o = ref.logprobs(v, tok, T, K)
        return (o["logprob"][0] * dl).sum() + (o["entropy"][0] * dh).sum() + (o["lse"][0] * dz).sum() + (o["top_logprob"][0] * dt).sum()
    got = ref.logprobs(x, tok, T, K, dl, dh, dz, dt, grad=True)
    agrees(f, x, got["dlogits"][0], g)


# ---- the C ABI ------------------------------------------------------------------------------


@pytest.fixture(scope="module")
def fe():
    import __graft_entry__
    __graft_entry__.build_lib_only()
    import paper_2509_20416_gb300 as fe
    return fe


MEMBERS = {  # each with the format characters before it
    "fe_project": dict(M=0, N=1, K=2, x=3, w=5, bias=7, residual=8, out=10, pre=12, act=14, work=16, work_bytes=17),
    "fe_project_backward": dict(M=0, N=1, K=2, x=3, w=5, dout=7, pre=9, dx=11, dw=13, dbias=15, act=16, work=18, work_bytes=19),
    "fe_gated_ffn": dict(M=0, F=1, K=2, x=3, w_gate=5, w_up=7, out=9, gate_pre=11, up_pre=13, act=15, work=17, work_bytes=18),
    "fe_gated_ffn_backward": dict(M=0, F=1, K=2, N=3, x=5, w_gate=7, w_up=9, w_down=11, dout=13, gate_pre=15, up_pre=17, dx=19, dw_gate=21,
                                  dw_up=23, dw_down=25, act=27, work=29, work_bytes=30),
    "fe_block_norm": dict(R=0, d=1, post=2, x=3, z=5, gate=7, gate_rows=9, post_w=10, pre_w=11, scale=12, offset=13, eps=14, y=16, n=18),
    "fe_block_norm_backward": dict(R=0, d=1, post=2, x=3, z=5, gate=7, gate_rows=9, post_w=10, pre_w=11, scale=12, offset=13, eps=14,
                                   dy=16, dn=18, dx=20, dz=22, dgate=24, dpost_w=26, dpre_w=27, work=28, work_bytes=29),
    "fe_token_logprobs": dict(R=0, V=1, J=2, K=3, logits=5, dtype=7, temperature=8, tokens=9, logprob=10, entropy=11, lse=12, stats=13,
                              top_id=14, top_logprob=15),
    "fe_token_logprobs_backward": dict(R=0, V=1, J=2, K=3, logits=5, dtype=7, temperature=8, tokens=9, top_id=10, stats=11, entropy=12,
                                       dlogprob=13, dentropy=14, dlse=15, dtop_logprob=16, dlogits=17),
}


def test_packed_arguments_match_the_header(fe, tmp_path):
    from paper_2509_20416_gb300 import layer
    assert set(MEMBERS) == set(layer._ARGS)
    src = ['#include <stdio.h>', '#include <stddef.h>', '#include "fe_layer.h"', 'int main(void) {']
    for f, ms in MEMBERS.items():
        src.append(f'printf("{f} %zu", sizeof({f}_args));')
        src += [f'printf(" %zu", offsetof({f}_args, {m}));' for m in ms]
        src.append('printf("\\n");')
    src.append('return 0; }')
    c = tmp_path / "offsets.c"
    c.write_text("\n".join(src))
    exe = str(tmp_path / "offsets")
    subprocess.run(["gcc", "-I" + os.path.join(ROOT, "include"), str(c), "-o", exe], check=True)
    for line in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines():
        f, size, *offsets = line.split()
        parts = []
        for n, k in re.findall(r"(\d*)([a-zA-Z])", layer._ARGS[f]):
            parts += [n + k] if k == "x" else [k] * int(n or 1)
        assert struct.calcsize("@" + layer._ARGS[f]) == int(size), f
        for m, off in zip(MEMBERS[f], offsets):
            n = MEMBERS[f][m]
            head = "@" + "".join(parts[:n]) + "0" + parts[n]
            assert struct.calcsize(head) == int(off), (f, m)


@pytest.fixture(scope="module")
def handle(fe):
    """The start of the library's handle (its configuration, device and number of SMs), which argument checks
    and the workspaces' sizes go by: they come before the GPU is asked for."""
    class Handle(ctypes.Structure):
        _fields_ = [("cfg", fe.target.fe_target_config), ("device", ctypes.c_int), ("num_sms", ctypes.c_int), ("rest", ctypes.c_byte * 64)]
    h = Handle(fe.make_target_config(dict(n_heads=1, n_kv_heads=1, head_dim=64, max_seq=16, dtype="f32", rope_theta=1e4)), 0, 152)
    return ctypes.addressof(h), h


P = 1 << 20  # an address that nothing reads


def good(name):
    m = lambda row=64: (P, row)
    none = (0, 0)
    return {
        "fe_project": [8, 64, 64, *m(), *m(), P, *m(), *m(), *none, 1, 0, 0],
        "fe_project_backward": [8, 64, 64, *m(), *m(), *m(), *m(), *m(), *m(), P, 1, P, 1 << 30],
        "fe_gated_ffn": [8, 64, 64, *m(), *m(), *m(), *m(), *none, *none, 2, 0, 0],
        "fe_gated_ffn_backward": [8, 64, 64, 64, *(m() * 11), 2, P, 1 << 30],
        "fe_block_norm": [8, 64, 1, *m(), *m(), *m(), 4, P, P, 1.0, 0.0, 1e-5, *m(), *m()],
        "fe_block_norm_backward": [8, 64, 1, *m(), *m(), *m(), 4, P, P, 1.0, 0.0, 1e-5, *(m() * 5), P, P, P, 1 << 30],
        "fe_token_logprobs": [8, 64, 2, 3, *m(), 0, 1.0, P, P, P, P, P, P, P],
        "fe_token_logprobs_backward": [8, 64, 2, 3, *m(), 0, 1.0, P, P, P, P, P, P, P, P, *m()],
    }[name]


def spoil(name, member, *values):
    """good(name) with a member's values changed, from its first one on (an index counts values, not padding)."""
    from paper_2509_20416_gb300 import layer
    chars = []
    for n, k in re.findall(r"(\d*)([a-zA-Z])", layer._ARGS[name]):
        chars += ["x"] if k == "x" else [k] * int(n or 1)
    at = sum(1 for k in chars[:MEMBERS[name][member]] if k != "x")
    v = good(name)
    v[at:at + len(values)] = values
    return v


SPOILT = {
    "fe_project": [("M", -1), ("M", 1 << 31), ("N", 0), ("K", 0), ("K", (1 << 24) + 1), ("act", 4), ("act", -1), ("x", 0), ("w", 0), ("out", 0),
                   ("x", P + 2), ("bias", P + 1), ("out", (P, 63)), ("x", (P, -64)), ("residual", P + 2)],
    "fe_project_backward": [("dout", 0), ("w", 0), ("x", 0), ("pre", 0), ("dx", (P, 63)), ("dw", (P, 0)), ("dbias", P + 2), ("N", 0),
                            ("work", 0), ("work", P + 16), ("work_bytes", 100), ("act", 9)],
    "fe_gated_ffn": [("gate_pre", P), ("up_pre", P), ("out", (P, 10)), ("w_up", 0), ("w_gate", 0), ("F", 0), ("act", 7), ("M", -5)],
    "fe_gated_ffn_backward": [("dw_up", 0), ("dw_gate", 0), ("w_up", 0), ("x", 0), ("gate_pre", 0), ("up_pre", 0), ("work_bytes", 0), ("w_down", 0), ("N", 0),
                              ("dw_down", (P, 63)),
                              ("dx", (P, 1)), ("dout", 0)],
    "fe_block_norm": [("R", -1), ("d", 0), ("z", 0), ("gate_rows", 0), ("scale", math.nan), ("offset", math.inf), ("eps", -1.0),
                      ("eps", math.nan), ("y", (P, 63)), ("n", (P, 1)), ("x", 0), ("post_w", P + 1), ("x", P + 1)],
    "fe_block_norm_backward": [("z", 0), ("gate_rows", 0), ("dx", (P, 3)), ("dgate", (P, 63)), ("work", 0), ("work_bytes", 255),
                               ("scale", math.inf), ("dpre_w", P + 3), ("gate", 0), ("post", 0)],
    "fe_token_logprobs": [("V", 0), ("J", 65), ("J", -1), ("K", 33), ("K", -1), ("V", 2), ("temperature", 0.0), ("temperature", math.nan),
                          ("temperature", -1.0), ("temperature", 1e-30), ("temperature", math.inf), ("dtype", 2), ("logits", 0),
                          ("tokens", 0), ("logprob", 0), ("top_id", 0), ("top_logprob", 0), ("R", -1), ("logits", P + 2)],
    "fe_token_logprobs_backward": [("stats", 0), ("tokens", 0), ("top_id", 0), ("entropy", 0), ("dlogits", 0), ("dlogits", (P, 63)),
                                   ("temperature", 0.0), ("logits", 0)],
}


@pytest.mark.parametrize("name", list(SPOILT))
def test_library_refuses_bad_arguments(fe, handle, name):
    """Refused by the checks that come before the device is looked at (here there is none)."""
    from paper_2509_20416_gb300 import layer
    call, size = getattr(fe._lib, name), layer._WORK.get(name)
    for member, value in SPOILT[name]:
        v = spoil(name, member, *(value if isinstance(value, tuple) else (value,)))
        packed = layer._PACK[name](*v)
        work = member.startswith("work")
        if not work:
            assert call(handle[0], packed, None) == fe.FE_ERR_INVALID_ARG, (member, value)
        if size is not None and not work:
            assert size(handle[0], packed) == fe.FE_ERR_INVALID_ARG, (member, value)
    packed = layer._PACK[name](*good(name))
    assert call(None, packed, None) == fe.FE_ERR_INVALID_ARG
    assert call(handle[0], None, None) == fe.FE_ERR_INVALID_ARG
    if size is not None:
        assert size(handle[0], packed) >= 0


def test_gates_of_more_rows_than_there_are(fe, handle):
    """A gate's rows may be any positive number: from R on they are one group."""
    from paper_2509_20416_gb300 import layer
    size = lambda rows, R: layer._WORK["fe_block_norm_backward"](
        handle[0], layer._PACK["fe_block_norm_backward"](*[R if i == 0 else v for i, v in enumerate(spoil("fe_block_norm_backward", "gate_rows", rows))]))
    for R in (1, 8, 5000):
        want = size(R, R)
        assert want > 0
        for rows in (R + 1, 1 << 31, 1 << 62, (1 << 63) - R, (1 << 63) - 1):
            assert size(rows, R) == want, (R, rows)
    assert size((1 << 63) - 1, 0) == 0


def test_binding_refuses_what_is_no_cuda_tensor(fe):
    t = fe.Target(0, dict(n_heads=1, n_kv_heads=1, head_dim=64, max_seq=16, dtype="f32", rope_theta=1e4))
    x, w = torch.zeros(2, 8), torch.zeros(4, 8)
    for call in (lambda: fe.fe_project(t, x, w), lambda: fe.fe_gated_ffn(t, x, w, w), lambda: fe.fe_block_norm(t, x, x),
                 lambda: fe.fe_token_logprobs(t, x, torch.zeros(2, dtype=torch.int32)),
                 lambda: fe.fe_project_backward(t, x, x=x, w=w.T), lambda: fe.fe_block_norm_backward(t, x, dy=x)):
        with pytest.raises(ValueError, match="CUDA|contiguous"):
            call()
    with pytest.raises(ValueError, match="residual"):
        fe.fe_gated_ffn(t, x, w, w, residual=x)
    with pytest.raises(ValueError, match="act"):
        fe.fe_project_backward(t, x, x=x, w=w, act="silu")
    with pytest.raises(ValueError, match="needs z"):
        fe.fe_block_norm(t, x, gate=x)
    with pytest.raises(ValueError, match="gate has"):
        fe.fe_block_norm(t, x, x, gate=x[:1], gate_rows=1)


def test_a_copy_on_a_stream_notes_its_source(fe, monkeypatch):
    """What a call copies on its stream is noted as in use there before the copy is queued: its memory may not be
    handed out again until the copy has run. Contiguous inputs are noted by the call itself."""
    from contextlib import nullcontext

    from paper_2509_20416_gb300 import layer
    monkeypatch.setattr(torch.cuda, "stream", lambda side: nullcontext())

    class Input:
        def __init__(self, contiguous):
            self.events, self._c = [], contiguous

        def is_contiguous(self):
            return self._c

        def record_stream(self, side):
            self.events.append(("in use", side))

        def contiguous(self):
            self.events.append("copy")
            return self
    x = Input(False)
    layer._contiguous(x, "side")
    assert x.events == [("in use", "side"), "copy"]
    x = Input(False)
    layer._contiguous(x, None)
    assert x.events == ["copy"]
    x = Input(True)
    assert layer._contiguous(x, "side") is x and not any(e != "copy" for e in x.events)


def test_a_block_with_outputs_given_is_not_recorded_in_part(fe, monkeypatch):
    """Outputs given keep a call out of autograd: its result must not carry the graph of the last product alone."""
    from paper_2509_20416_gb300 import layer
    seen = []
    monkeypatch.setattr(layer, "_mat", lambda x, dtype, shape: (0, 0))
    monkeypatch.setattr(layer, "_call", lambda name, t, side, tensors, args: seen.append((name, tensors)))
    t = fe.Target(0, dict(n_heads=1, n_kv_heads=1, head_dim=64, max_seq=16, dtype="f32", rope_theta=1e4))
    x, wg, wu, wd, r = (torch.zeros(8, 8, requires_grad=True) for _ in range(5))
    for given in (dict(gate_pre=torch.empty(8, 8), up_pre=torch.empty(8, 8)), dict(out=torch.empty(8, 8)),
                  dict(out=torch.empty(8, 8), gate_pre=torch.empty(8, 8), up_pre=torch.empty(8, 8))):
        seen.clear()
        y = fe.fe_gated_ffn(t, x, wg, wu, wd, residual=r, **given)
        assert not y.requires_grad, list(given)
        assert [name for name, _ in seen] == ["fe_gated_ffn", "fe_project"]
        assert not seen[1][1][0].requires_grad, list(given)  # (h)
    assert fe.fe_gated_ffn(t, x, wg, wu, wd, residual=r).requires_grad


def test_outputs_given_count_as_changed(fe, monkeypatch):
    """Autograd learns of what the kernels write into a caller's tensors, by their versions."""
    from paper_2509_20416_gb300 import layer, target
    monkeypatch.setattr(layer, "_mat", lambda x, dtype, shape: (0, 0))
    monkeypatch.setattr(layer, "_call", lambda name, t, side, tensors, args: None)
    for f in ("_rows", "_ints"):
        monkeypatch.setattr(target, f, lambda *a: (0, 0, 0, 0) if len(a) == 3 else 0)
    monkeypatch.setattr(target, "_call", lambda *a: None)
    t = fe.Target(0, dict(n_heads=1, n_kv_heads=1, head_dim=8, max_seq=16, dtype="f32", rope_theta=1e4))
    x, w = torch.zeros(8, 8), torch.zeros(8, 8)
    q, pos = torch.zeros(2, 4, 1, 8), torch.zeros(2, 4, dtype=torch.int32)

    class Flat:  # (a cache)
        def _layer(self, i, B):
            return ()
    new = lambda like=x: torch.zeros_like(like)
    calls = [lambda a, b: fe.fe_project(t, x, w, out=a, pre=b), lambda a, b: fe.fe_gated_ffn(t, x, w, w, gate_pre=a, up_pre=b),
             lambda a, b: (fe.fe_gated_ffn(t, x, w, w, w, out=a), fe.fe_gated_ffn(t, x, w, w, out=b)),
             lambda a, b: fe.fe_block_norm(t, a, x, y=a, n=b)]
    for i, call in enumerate(calls):
        a, b = new(), new()
        call(a, b)
        assert a._version > 0 and b._version > 0, i
    assert x._version == 0 and w._version == 0
    for i, call in enumerate([lambda a, b: fe.fe_rope(t, a, b, pos, q_out=a, k_out=b),
                              lambda a, b: (fe.fe_cache_write(t, Flat(), 0, q, q, pos[:, 0], q=q, q_out=a), fe.fe_rope(t, b, None, pos, q_out=b)),
                              lambda a, b: fe.fe_cache_read(t, Flat(), 0, pos[:, 0], None, 4, a, b)]):
        a, b = new(q), new(q)
        call(a, b)
        assert a._version > 0 and b._version > 0, i
    with torch.inference_mode():
        y = torch.zeros(8, 8)
    fe.fe_project(t, x, w, out=y)  # (has no version)


def test_row_strides(fe):
    from paper_2509_20416_gb300.layer import _row
    x = torch.zeros(4, 6, 10)
    assert _row(x) == 10 and _row(x[:, :, 2:5]) == 10 and _row(x[:1, :1]) == 0 and _row(x[:, ::2]) == 20
    assert _row(x[:, :3]) is None and _row(x.transpose(0, 1)) is None and _row(x.transpose(1, 2)) is None
    assert _row(x[0, 0]) == 0 and _row(x[:1].expand(4, 6, 10)) is None and _row(x[0, :1].expand(7, 10)) == 0
