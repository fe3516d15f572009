"""Corners of the target-side operators on the GPU, against the plain 64-bit forms (target_ref.py)
and with the bounds of test_gpu_target.py, unless a test derives its own."""
import math

import pytest
import torch

import target_ref as ref
from test_gpu_target import check_attention, gen

pytestmark = pytest.mark.gpu

TYPES = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "e4m3")]


@pytest.fixture(scope="module")
def fe():
    import paper_2509_20416_gb300 as fe
    return fe


def fill(store, name, rows, cache):
    """Rows [heads, slots, hd] (float) into layer 0 of a contiguous cache of one sequence."""
    if cache == "e4m3":
        e, s = ref.quantise(rows)
        getattr(store, name)[0, 0, :, :rows.shape[1]] = e.to(torch.float8_e4m3fn).cuda()
        getattr(store, name + "_scale")[0, 0, :, :rows.shape[1]] = s.float().cuda()
    else:
        getattr(store, name)[0, 0, :, :rows.shape[1]] = rows.to(ref.DT[cache]).cuda()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("H,Hkv,hd,T", [(2, 2, 128, 5), (4, 2, 64, 40), (8, 2, 128, 60), (4, 1, 64, 70)])
def test_maximum_that_grows_at_every_step(fe, dtype, cache, H, Hkv, hd, T):
    """A row's maximum grows by 10 (a factor of 2^14.4) at every 32nd slot, so that running sums,
    probabilities and outputs are rescaled several times within a tile, directly after they were
    written; values shrink as the probabilities grow, so that every step of the last two tiles weighs
    the same in the result. Rows of four kinds: growing, shrinking, every second step, none."""
    steps, P = 24, 24 * 32 - T
    c = ref.config(dtype=dtype, cache_dtype=cache, n_heads=H, n_kv_heads=Hkv, head_dim=hd, max_batch=1, max_seq=1024)
    t = fe.fe_target_init(c)
    g = gen(T + hd)
    store = ref.random_cache(fe, t, c, g)
    step = torch.arange(P + T) // 32
    k = torch.zeros(Hkv, P + T, hd)
    k[:, torch.arange(P + T), step] = 1.0  # a slot's score: the query's element of its step
    v = torch.randn(Hkv, P + T, hd, generator=g) * torch.exp2(-14.0 * (step % 8))[:, None]
    fill(store, "k", k, cache)
    fill(store, "v", v, cache)
    s = torch.arange(steps)
    kinds = torch.stack([10 * s, 10 * (steps - s), 20 * (s // 2), 50 * torch.ones_like(s)]).float()
    q = torch.zeros(1, T, H, hd)
    for i in range(T):
        for h in range(H):
            q[0, i, h, :steps] = kinds[(i + h) % 4 if T > 5 else 0]
    q = q.to(ref.DT[dtype]).cuda()
    plen = torch.tensor([P], dtype=torch.int32)
    out, lse = fe.fe_tree_attention(t, store, 0, q, plen.cuda(), scale=1.0)
    assert fe.fe_target_status(t) == fe.FE_OK
    check_attention(c, store, None, q, plen, torch.tensor([T]), None, out, lse, scale=1.0)
