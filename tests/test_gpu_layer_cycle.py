"""The whole cycle of examples/verify_cycle.py with a target of whole layers on the dense operators: text
decoded through draft trees is the text decoded token by token. float32 passes over a tree and over single
tokens agree to some 1e-6 of the logits, far below the gaps between a random head's largest logits;
16- and 8-bit caches round alike up to the order of sums, so that texts may part at a near-tie but not at
once."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cycle():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import verify_cycle
    return verify_cycle


@pytest.mark.parametrize("cache", ["f32", "bf16", "e4m3"])
def test_text_of_whole_layers(cycle, cache):
    text, plain, accepted = cycle.run(cache, 20, target="layers")
    for t, p in zip(text, plain):
        assert t == p if cache == "f32" else t[:3] == p[:3]
    assert sum(sum(a) for a in accepted) > 0


@pytest.mark.parametrize("cache", ["f32", "bf16"])
def test_forward_of_a_layer_target(cycle, cache):
    """One pass over a ragged prompt against the same layers in float64: features within a share of their
    norm that the roundings of a pass explain (some twenty of them, each half a step of the type)."""
    import paper_2509_20416_gb300 as fe
    from fe_synth import workloads as wl
    cfg = wl.make_config("tiny", B=2, max_seq=64)
    W = wl.make_weights(cfg)
    t = cycle.LayerTarget(cfg, W, cache, 2, 64)
    g = torch.Generator().manual_seed(3)
    tok, n = cycle.pad([torch.randint(0, cfg["vocab"], (k,), generator=g).tolist() for k in (9, 5)])
    pos = torch.arange(9, dtype=torch.int32, device="cuda").repeat(2, 1)
    nxt, feat = t.forward(tok, pos, torch.zeros(2, dtype=torch.int32, device="cuda"), n_rows=n)
    assert fe.fe_target_status(t.t) == fe.FE_OK
    norm = lambda a, w: a * (a.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w.double()
    H, hd = t.H, t.hd
    x = (t.embed[tok.long()] * 50.0).double()
    states = [x]
    f = cfg["rope_theta"] ** (-torch.arange(0, hd, 2, dtype=torch.float64, device="cuda") / hd)
    ang = pos.double()[..., None] * f
    cos, sin = ang.cos()[:, :, None], ang.sin()[:, :, None]

    def turn(v):
        a, b = v[..., :hd // 2], v[..., hd // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    for L in t.layers:
        u = norm(x, L["attn_norm"])
        q, k, v = (u @ L["qkv"].double().T).view(2, 9, 3 * H, hd).split([H, H, H], 2)
        s = torch.einsum("bihd,bjhd->bhij", turn(q), turn(k)) / hd ** 0.5
        s = s.masked_fill(~torch.ones(9, 9, device="cuda").tril().bool(), float("-inf"))
        a = torch.einsum("bhij,bjhd->bihd", torch.softmax(s, -1), v).reshape(2, 9, -1)
        x = x + norm(a @ L["o"].double().T, L["post_norm"])
        u = norm(x, L["mlp_norm"])
        x = x + (torch.nn.functional.silu(u @ L["gate"].double().T) * (u @ L["up"].double().T)) @ L["down"].double().T
        states.append(x)
    want = torch.cat([states[0], states[1], states[-1]], -1)
    unit = 2.0 ** -24 * 64 if cache == "f32" else 2.0 ** -8
    for b in range(2):
        got = feat[b, :n[b]].double()
        assert (got - want[b, :n[b]]).norm() <= 20 * unit * want[b, :n[b]].norm()
    if cache == "f32":
        logits = norm(x, t.final_norm) @ t.head.double().T
        for b in range(2):
            assert torch.equal(nxt[b, :n[b]].long(), logits[b, :n[b]].argmax(-1))
