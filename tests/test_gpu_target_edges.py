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


@pytest.fixture(scope="module")
def join(tmp_path_factory):
    """The join kernel alone (tests/cuda/join_notes.cu)."""
    import ctypes
    import os
    import subprocess
    from paper_2509_20416_gb300 import build
    here = os.path.dirname(os.path.abspath(__file__))
    lib = str(tmp_path_factory.mktemp("join") / "join_notes.so")
    subprocess.run([build.nvcc(), *build.ARCH, *build.NVCC_FLAGS, "-shared", os.path.join(here, "cuda", "join_notes.cu"),
                    "-o", lib], check=True, capture_output=True, text=True)
    so = ctypes.CDLL(lib)

    def run(notes, part_o, part_ml, T=5, ncta=4):
        """notes: (b, h, m, rows, last, has0) of each CTA; returns out [T, 2, 64], lse [T, 2] and what
        lies before and behind them."""
        assert so.note_bytes() == 32
        out, lse = torch.full((3, T, 2, 64), 7.0, device="cuda"), torch.full((3, T, 2), 7.0, device="cuda")
        d = torch.tensor([list(n) + [0, 0] for n in notes], dtype=torch.int32, device="cuda")
        ints = torch.zeros(2, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        p = lambda x: ctypes.c_void_p(x.data_ptr())
        assert so.join_notes(T, ncta, p(out[1]), p(lse[1]), p(ints), p(d), p(part_o), p(part_ml), p(ints[1:])) == 0
        assert (out[[0, 2]] == 7.0).all() and (lse[[0, 2]] == 7.0).all()
        return out[1], lse[1]
    return run


def test_join_stays_within_the_grid(join):
    """Notes as a first call finds them, as a CTA leaves them that gave up, and one that names CTAs
    beyond the grid: nothing is written, or the item's shares inside the grid are joined."""
    g, T, ncta = gen(3), 5, 4
    part_o = torch.randn(2 * ncta, 16, 64, 4, generator=g).cuda()  # [CTA and slot][columns / 4][row][4]
    part_ml = torch.stack([torch.randn(2 * ncta, 64, generator=g), torch.rand(2 * ncta, 64, generator=g) + 0.5], -1).cuda()
    none = (0, 0, 0, 0, -1, 0)
    for notes in ([(0, 0, 0, 0, 0, 0)] * ncta, [none] * ncta, [(0, 0, 0, T, -1, 1)] * ncta):
        out, lse = join(notes, part_o, part_ml)
        assert (out == 7.0).all() and (lse == 7.0).all()
    for last in (3, 4, 1 << 20, 2**31 - 1):  # shares: CTA 1's slot 1, CTA 3's slot 0 (CTA 2 has none)
        out, lse = join([none, (0, 1, 0, T, last, 0), (0, 0, 0, 0, -1, 0), (0, 0, 0, 0, -1, 1)], part_o, part_ml)
        assert (out[:, 0] == 7.0).all() and (lse[:, 0] == 7.0).all()
        m, l = part_ml[[3, 6], :T].double().unbind(-1)
        w = torch.exp2(m - m.amax(0))
        o = part_o[[3, 6]].double().permute(0, 2, 1, 3).reshape(2, 64, 64)[:, :T]
        want = (w[..., None] * o).sum(0) / (w * l).sum(0)[:, None]
        # two products, a sum and a quotient in float32, and 2^x: a few roundings of what is summed
        size = (w[..., None] * o.abs()).sum(0) / (w * l).sum(0)[:, None]
        assert ((out[:, 1].double() - want).abs() <= 2.0 ** -19 * size).all()
        assert ((lse[:, 1].double() - (m.amax(0) * math.log(2) + torch.log((w * l).sum(0)))).abs() <= 2.0 ** -19).all()
