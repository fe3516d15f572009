"""Corners of the target-side operators on the GPU, against the plain 64-bit forms (target_ref.py)
and with the bounds of test_gpu_target.py, unless a test derives its own."""
import math

import pytest
import torch

import target_ref as ref
from test_gpu_target import check_attention, gen, tree_masks

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


def classes(x):
    """0 finite, 1 NaN, 2 +inf, 3 -inf."""
    return torch.isnan(x) * 1 + (x == math.inf) * 2 + (x == -math.inf) * 3


def check_classes(c, store, q, P, n, mask, out, lse):
    """Outputs and log-sum-exps are finite, NaN, +inf or -inf exactly where the 64-bit form's are."""
    H, Hkv, hd = c["n_heads"], c["n_kv_heads"], c["head_dim"]
    G = H // Hkv
    for b in range(q.shape[0]):
        nb, Pb = int(n[b]), int(P[b])
        see = torch.ones(nb, Pb + nb, dtype=torch.bool, device="cuda")
        see[:, Pb:] = (mask[b, :nb, :nb].cuda() != 0) if mask is not None else torch.ones(nb, nb, device="cuda").tril().bool()
        for h in range(Hkv):
            k, v = ref.cache_rows(c, store, 0, b, h, Pb + nb)
            for gq in range(G):
                o, l, _, _ = ref.attend(q[b, :nb, h * G + gq], k, v, see, 1 / math.sqrt(hd))
                assert torch.equal(classes(out[b, :nb, h * G + gq]), classes(o)), (b, h, gq)
                assert torch.equal(classes(lse[b, :nb, h * G + gq]), classes(l)), (b, h, gq)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("T,P", [(9, [40, 90]), (40, [100, 300]), (70, [3000]), (140, [10, 700])])
def test_infinities_of_prefix_and_nodes_meet(fe, dtype, cache, T, P):
    """Values of +inf, -inf and NaN in the prefix and in nodes that some nodes see, in the same column
    and in different ones: opposite infinities and NaN give NaN, alone they stay what they are."""
    B, H, Hkv, hd = len(P), 4, 2, 128
    c = ref.config(dtype=dtype, cache_dtype=cache, n_heads=H, n_kv_heads=Hkv, head_dim=hd, max_batch=B, max_seq=max(P) + T + 1)
    t = fe.fe_target_init(c)
    g = gen(T)
    store = ref.random_cache(fe, t, c, g)
    inf, nan = (math.inf, math.nan) if cache != "e4m3" else (math.nan, math.nan)
    near, far = [p - 1 for p in P], [p // 7 for p in P]  # prefix slots: the nodes' tile as a rule, and an early one
    for b in range(B):
        v = store.v[0, b]
        # columns: prefix alone (0-3), nodes alone (8-10), both (16-23)
        for h in range(Hkv):
            for col, slot, x in ((0, near[b], inf), (1, far[b], -inf), (2, near[b], nan), (3, far[b], nan),
                                 (8, P[b] + 1, inf), (9, P[b] + 3, -inf), (10, P[b] + 4, nan),
                                 (16, near[b], inf), (16, P[b] + 1, -inf), (17, far[b], inf), (17, P[b] + 3, -inf),
                                 (18, near[b], nan), (18, P[b] + 1, -inf), (19, far[b], -inf), (19, P[b] + 1, -inf),
                                 (20, far[b], nan), (20, P[b] + 4, inf), (21, P[b] + 1, inf), (21, P[b] + 3, -inf),
                                 (22, near[b], inf), (22, P[b] + 4, nan), (23, near[b], inf), (23, P[b] + 3, inf)):
                v[h, slot, col + 64 * h] = x
    # every second node sees node 1, every third node 3, every fifth node 4
    mask = torch.zeros(B, T, T, dtype=torch.uint8)
    i = torch.arange(T)
    for node, every in ((1, 2), (3, 3), (4, 5)):
        mask[:, i % every == 0, node] = 1
    mask[:, i, i] |= torch.tensor([0 if j in (1, 3, 4) else 1 for j in range(T)], dtype=torch.uint8)
    # scores stay small: no probability rounds to zero
    q = (0.3 * torch.randn(B, T, H, hd, generator=g)).to(ref.DT[dtype]).cuda()
    plen = torch.tensor(P, dtype=torch.int32)
    out, lse = fe.fe_tree_attention(t, store, 0, q, plen.cuda(), mask=mask.cuda())
    assert fe.fe_target_status(t) == fe.FE_OK
    assert torch.isnan(out).any() and (cache == "e4m3" or torch.isinf(out).any())
    check_classes(c, store, q, P, [T] * B, mask, out, lse)
    check_attention(c, store, None, q, plen, torch.tensor([T] * B), mask, out, lse)


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("dtype,cache", TYPES)
def test_a_prompt_of_non_finite_values_takes_no_time(fe, dtype, cache, value):
    """A chunk whose values are all NaN, or all infinite (NaN in an e4m3 cache): right by kind, and in
    some milliseconds at most, far below the two seconds after which a wait inside the kernel runs
    out. (A pass over all slots for each of a row's columns took half a second.)"""
    T, P, H, hd = 600, 70, 2, 128
    c = ref.config(dtype=dtype, cache_dtype=cache, n_heads=H, n_kv_heads=1, head_dim=hd, max_batch=1, max_seq=P + T)
    t = fe.fe_target_init(c)
    g = gen(T)
    store = ref.random_cache(fe, t, c, g)
    q = (0.3 * torch.randn(1, T, H, hd, generator=g)).to(ref.DT[dtype]).cuda()
    plen = torch.tensor([P], dtype=torch.int32).cuda()
    fe.fe_tree_attention(t, store, 0, q, plen)
    store.v[0, 0, :, P:] = math.nan if cache == "e4m3" else value
    store.v[0, 0, :, P + 100:P + 300, 5] = 1.0  # (finite, alone of their rows)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    out, lse = fe.fe_tree_attention(t, store, 0, q, plen)
    end.record()
    assert fe.fe_target_status(t) == fe.FE_OK
    check_classes(c, store, q, [P], [T], None, out, lse)
    assert begin.elapsed_time(end) < 50.0


@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("bf16", "bf16")])
def test_an_infinite_value_at_probability_zero(fe, dtype, cache):
    """A node whose key makes a score of -inf has probability zero: its infinite values give NaN, as
    zero times infinity does, and its finite ones nothing."""
    T, P, hd = 33, 20, 64
    c = ref.config(dtype=dtype, n_heads=2, n_kv_heads=1, head_dim=hd, max_batch=1, max_seq=P + T)
    t = fe.fe_target_init(c)
    g = gen(T)
    store = ref.random_cache(fe, t, c, g)
    q = (0.3 * torch.randn(1, T, 2, hd, generator=g)).abs().to(ref.DT[dtype]).cuda()
    store.k[0, 0, 0, P + 3, 7] = -math.inf
    store.v[0, 0, 0, P + 3, 1] = math.inf
    store.v[0, 0, 0, P + 4, 2] = -math.inf
    plen = torch.tensor([P], dtype=torch.int32)
    out, lse = fe.fe_tree_attention(t, store, 0, q, plen.cuda())
    assert fe.fe_target_status(t) == fe.FE_OK
    assert torch.isnan(out[0, 3:, :, 1]).all() and (out[0, 4:, :, 2] == -math.inf).all()
    check_classes(c, store, q, [P], [T], None, out, lse)
    check_attention(c, store, None, q, plen, torch.tensor([T]), None, out, lse)


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("call", ["rope", "write", "read", "attention"])
def test_new_outputs_on_another_stream_are_not_written_early(fe, call, handle):
    """Memory just freed on the current stream, which kernels queued there still write, is not handed
    out as the output of a call that runs at once on another stream."""
    T, H, hd = 256, 64, 128
    c = ref.config(n_heads=H, n_kv_heads=H, max_batch=1, max_seq=512)
    t = fe.fe_target_init(c)
    g = gen(1)
    store = ref.random_cache(fe, t, c, g)
    q, k = (torch.randn(1, T, H, hd, generator=g).bfloat16().cuda() for _ in range(2))
    pos = torch.arange(T, dtype=torch.int32)[None].cuda()
    zero, n = torch.zeros(1, dtype=torch.int32).cuda(), torch.full((1,), T, dtype=torch.int32).cuda()
    run = {"rope": lambda **kw: fe.fe_rope(t, q, None, pos, **kw)[0],
           "write": lambda **kw: fe.fe_cache_write(t, store, 0, k, k, zero, pos=pos, q=q, **kw),
           "read": lambda **kw: fe.fe_cache_read(t, store, 0, zero, n, T, **kw)[0],
           "attention": lambda **kw: fe.fe_tree_attention(t, store, 0, q, zero, **kw)[0]}[call]
    want = run().clone()
    other = torch.full_like(want, 3.0)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    freed = torch.empty_like(want)
    torch.cuda._sleep(1_000_000_000)
    freed.copy_(other)  # (runs after the pause)
    del freed
    got = run(stream=s.cuda_stream if handle else s)
    s.synchronize()
    assert not torch.cuda.current_stream().query()  # the pause is still going on
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    assert fe.fe_target_status(t) == fe.FE_OK


def test_status_is_read_and_cleared_on_its_own_stream(fe):
    """fe_target_status(stream) neither waits for another stream's work, the default stream's
    included, nor clears an error of a call that follows it on the same stream."""
    c = ref.config(max_batch=1, max_seq=32)
    t = fe.fe_target_init(c)
    store = fe.alloc_cache(t, 1)
    k = torch.zeros(1, 1, 2, 128, dtype=torch.bfloat16, device="cuda")
    bad, good = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (99, 3))
    s = torch.cuda.Stream()
    fe.fe_cache_write(t, store, 0, k, k, good)  # (a first launch loads its kernel, which may wait for others)
    assert fe.fe_target_status(t) == fe.FE_OK
    torch.cuda.synchronize()
    torch.cuda._sleep(1_000_000_000)
    fe.fe_cache_write(t, store, 0, k, k, bad, stream=s)
    assert fe.fe_target_status(t, stream=s) == fe.FE_ERR_CAPACITY
    for _ in range(20):
        fe.fe_cache_write(t, store, 0, k, k, good, stream=s)
        assert fe.fe_target_status(t, stream=s) == fe.FE_OK
        fe.fe_cache_write(t, store, 0, k, k, bad, stream=s)
        assert fe.fe_target_status(t, stream=s) == fe.FE_ERR_CAPACITY
    assert not torch.cuda.current_stream().query()  # the default stream's pause is still going on
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_positions_of_rows_that_are_not_written(fe, dtype, cache):
    """Without queries, the positions of rows from n_rows[b] on (padding of ragged trees) may be
    anything; a bad position of a row that is written is reported, and that row skipped."""
    c = ref.config(dtype=dtype, cache_dtype=cache, max_batch=2, max_seq=64)
    t = fe.fe_target_init(c)
    store = fe.alloc_cache(t, 1)
    k = torch.randn(2, 5, 2, 128, generator=gen(1)).to(ref.DT[dtype]).cuda()
    start, n = torch.tensor([7, 20], dtype=torch.int32).cuda(), torch.tensor([2, 4], dtype=torch.int32).cuda()
    pos = torch.tensor([[7, 8, -1, 64, 2**31 - 1], [20, 21, 22, 21, -9]], dtype=torch.int32).cuda()
    fe.fe_cache_write(t, store, 0, k, k, start, n_rows=n, pos=pos)
    assert fe.fe_target_status(t) == fe.FE_OK
    written = (store.v[0].float() != 0).any(-1).nonzero().tolist()
    assert written == [[0, h, s] for h in range(2) for s in (7, 8)] + [[1, h, s] for h in range(2) for s in (20, 21, 22, 23)]
    store.v.zero_()
    pos[0, 1] = -1
    fe.fe_cache_write(t, store, 0, k, k, start, n_rows=n, pos=pos)
    assert fe.fe_target_status(t) == fe.FE_ERR_CAPACITY
    written = (store.v[0].float() != 0).any(-1).nonzero().tolist()
    assert written == [[0, h, 7] for h in range(2)] + [[1, h, s] for h in range(2) for s in (20, 21, 22, 23)]
    fe.fe_cache_write(t, store, 0, k, k, start, n_rows=torch.tensor([-1, 6], dtype=torch.int32).cuda(), pos=pos.clamp(0, 9))
    assert fe.fe_target_status(t) == fe.FE_ERR_DEVICE


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout,scaling", [("half", "none"), ("interleaved", "yarn")])
def test_rope_under_autograd(fe, dtype, layout, scaling):
    """Rotations of tensors that require gradients are differentiable: the gradient is the transposed
    rotation, checked against its 64-bit form (the bound of test_gpu_target.py: 4 * 2^-24 of amplitude
    * (|a| + |b|), and u |y|) and, for float32, against differences. The map is linear, so a central
    difference of sum(y g) has no error but its roundings: with x and x + d rounded to float32 and
    sums in 64 bits, each y is off by 4 * 2^-24 (|a| + |b|) amp + 2^-24 |y| on either side."""
    c = ref.config(dtype=dtype, rope_layout=layout, rope_scaling=scaling, rope_dim=96, rope_factor=4.0, rope_orig=128.0,
                   rope_low=32.0, rope_high=1.0)
    t = fe.fe_target_init(c)
    g, u = gen(5), ref.UNIT[dtype]
    B, T, dt = 2, 7, ref.DT[dtype]
    leaf = [torch.randn(B, T, n, 128, generator=g).to(dt).cuda().requires_grad_() for n in (8, 2)]
    pos = torch.randint(0, 512, (B, T), generator=g, dtype=torch.int32).cuda()
    grads = [torch.randn(B, T, n, 128, generator=g).to(dt).cuda() for n in (8, 2)]
    out = fe.fe_rope(t, *leaf, pos)
    plain = fe.fe_rope(t, *(x.detach() for x in leaf), pos)
    assert all(o.requires_grad and torch.equal(o, p) for o, p in zip(out, plain))
    got = torch.autograd.grad(out, leaf, grads)
    for x, d in zip(got, grads):
        want, mag = ref.rotate(c, d, pos, backward=True)
        assert ((x.double() - want).abs() <= 4 * 2.0 ** -24 * mag + u * want.abs()).all()
    # one input alone; a gradient with strides of zero; the gradient's own gradient
    k = leaf[1]
    none, ko = fe.fe_rope(t, None, k, pos)
    assert none is None
    ones, _ = ref.rotate(c, torch.ones_like(k), pos, backward=True)
    dk, = torch.autograd.grad(ko.sum(), k)
    assert ((dk.double() - ones).abs() <= (8 * 2.0 ** -24 * 2 * 1.2 + u * ones.abs())).all()
    w = grads[1].clone().requires_grad_()
    dk, = torch.autograd.grad(fe.fe_rope(t, None, k, pos)[1], k, w, create_graph=True)
    back, = torch.autograd.grad(dk, w, grads[1])
    assert torch.equal(back, fe.fe_rope(t, None, grads[1], pos)[1])
    # q's graph only: k stays outside it
    qo, ko = fe.fe_rope(t, leaf[0], k.detach(), pos)
    dq, = torch.autograd.grad(qo, leaf[0], grads[0])
    assert torch.equal(dq, got[0])
    with torch.no_grad():
        assert not fe.fe_rope(t, *leaf, pos)[0].requires_grad
    if dtype == "f32":
        for x, d, dx, n in zip(leaf, grads, got, range(2)):
            e = torch.randn(x.shape, generator=g).cuda()
            a, b = (x + e).detach(), (x - e).detach()
            ya, yb = (fe.fe_rope(t, *((z, None) if n == 0 else (None, z)), pos)[n] for z in (a, b))
            diff = ((ya.double() - yb.double()) * d.double()).sum()
            want = ((a.double() - b.double()) * dx.double()).sum()
            tol = sum(((5 * 2.0 ** -24 * ref.rotate(c, z, pos)[1]) * d.double().abs()).sum() for z in (a, b)) \
                + ((a - b).double().abs() * (5 * 2.0 ** -24 * ref.rotate(c, d, pos, backward=True)[1])).sum()
            assert (diff - want).abs() <= tol


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("page", [0, 16])
def test_calls_captured_in_a_graph(fe, dtype, cache, page):
    """A step's calls captured once and replayed on new inputs, lengths and counts give the bits of
    direct calls."""
    B, T, H, Hkv, hd = 3, 21, 8, 2, 128
    c = ref.config(dtype=dtype, cache_dtype=cache, n_heads=H, n_kv_heads=Hkv, head_dim=hd, page_size=page, max_batch=B, max_seq=512)
    t = fe.fe_target_init(c)
    g = gen(page)
    table, n_pages = ref.paged(c, B, g)
    store, twin = (ref.random_cache(fe, t, c, gen(page + 1), layers=2, table=table, n_pages=n_pages) for _ in range(2))
    qkv = torch.zeros(B, T, H + 2 * Hkv, hd, dtype=ref.DT[dtype], device="cuda")
    q, k, v = qkv.split([H, Hkv, Hkv], 2)
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    start, n, pos, path, acc = ints(B), ints(B), ints(B, T), ints(B, 3), ints(B)
    mask = torch.zeros(B, T, T, dtype=torch.uint8, device="cuda")

    def step(cache):
        r = fe.fe_cache_write(t, cache, 1, k, v, start, n_rows=n, pos=pos, q=q)
        out, lse = fe.fe_tree_attention(t, cache, 1, r, start, mask=mask, n_nodes=n)
        fe.fe_cache_keep(t, cache, path, acc, start)
        return r, out, lse, *fe.fe_cache_read(t, cache, 1, start, n, T)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(store)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(store)
    for x in ("k", "v", "k_scale", "v_scale"):  # (the warm-up wrote a row)
        if getattr(store, x) is not None:
            getattr(store, x).view(torch.uint8).copy_(getattr(twin, x).view(torch.uint8))
    for i in range(3):
        P = torch.randint(0, 512 - T, (B,), generator=g, dtype=torch.int32)
        for to, x in ((qkv, torch.randn(qkv.shape, generator=g)), (start, P), (n, torch.randint(4, T + 1, (B,), generator=g)),
                      (pos, P[:, None] + torch.arange(T)), (mask, tree_masks(g, B, T)), (path, torch.tensor([[1, 2, 3]] * B)),
                      (acc, torch.randint(0, 4, (B,), generator=g))):
            to.copy_(x.to(to.dtype))
        graph.replay()
        want = step(twin)
        assert fe.fe_target_status(t) == fe.FE_OK
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want)), i
        assert torch.equal(store.k.view(torch.uint8), twin.k.view(torch.uint8))


@pytest.mark.parametrize("size", [2.0 ** 5, 2.0 ** 10, 2.0 ** 14])
@pytest.mark.parametrize("T", [6, 50])
def test_queries_with_an_outlier_over_e4m3(fe, T, size):
    """One element of a query row far above the rest, met by small key elements. Over e4m3 a query
    element is exact down to 2^-10 of the scale 2^c, the smallest with the row's largest magnitude
    below 448 times it, and off by 2^-10 2^c at most; a score by f = scale 2^-10 2^c sum |k|. So every
    probability carries a relative error below e + exp(2 f) - 1 (e as in test_gpu_target.py), and the
    log-sum-exp one of f."""
    H, Hkv, hd, P = 4, 2, 128, 300
    c = ref.config(cache_dtype="e4m3", n_heads=H, n_kv_heads=Hkv, head_dim=hd, max_batch=1, max_seq=P + T)
    t = fe.fe_target_init(c)
    g = gen(T)
    store = ref.random_cache(fe, t, c, g)
    for name in ("k", "v"):
        x = torch.randn(Hkv, P + T, hd, generator=g)
        if name == "k":
            x[..., 77] *= 2.0 ** -8
        fill(store, name, x, "e4m3")
    q = torch.randn(1, T, H, hd, generator=g)
    q[..., 77] = size * torch.sign(q[..., 77])
    q = q.bfloat16().cuda()
    scale = 1 / math.sqrt(hd)
    out, lse = fe.fe_tree_attention(t, store, 0, q, torch.tensor([P], dtype=torch.int32).cuda())
    assert fe.fe_target_status(t) == fe.FE_OK
    see = torch.ones(T, P + T, device="cuda").tril(P).bool()
    for h in range(Hkv):
        k, v = ref.cache_rows(c, store, 0, 0, h, P + T)
        for i in range(h * 2, h * 2 + 2):
            o, l, mag, A = ref.attend(q[0, :, i], k, v, see, scale)
            c2 = torch.ceil(torch.log2(q[0, :, i].double().abs().amax(-1) / 448))
            f = scale * 2.0 ** -10 * torch.exp2(c2) * k.abs().sum(-1).amax()
            e = 2 * (hd + 4) * 2.0 ** -24 * A + 2.0 ** -20
            tol = ((e + torch.expm1(2 * f))[:, None] + 1.01 * 2.0 ** -8) * mag + 2.0 ** -8 * o.abs()
            assert ((out[0, :, i].double() - o).abs() <= tol).all()
            assert ((lse[0, :, i].double() - l).abs() <= e + f + 2.0 ** -23 * l.abs()).all()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("T", [30, 90])
def test_probabilities_are_rounded_once(fe, cache, T):
    """A slot at the start of a tile in which the maximum then grows three times by 2^13 to 2^20: its
    probability is all that half of the columns see. It may be off by one rounding to bfloat16, as in
    test_gpu_target.py's bound, however often the row's reference moves."""
    H, Hkv, hd, P = 8, 2, 128, 128
    c = ref.config(cache_dtype=cache, n_heads=H, n_kv_heads=Hkv, head_dim=hd, max_batch=1, max_seq=P + T)
    t = fe.fe_target_init(c)
    g = gen(T)
    store = ref.random_cache(fe, t, c, g)
    k = torch.zeros(Hkv, P + T, hd)
    k[:, torch.arange(P), torch.arange(P) // 32] = 1.0
    v = torch.randn(Hkv, P + T, hd, generator=g)
    v[:, 1:, :64] = 0.0
    fill(store, "k", k, cache)
    fill(store, "v", v, cache)
    q = torch.zeros(1, T, H, hd)
    q[..., :4] = (9 + 5 * torch.rand(1, T, H, 4, generator=g)).cumsum(-1)
    q = q.bfloat16().cuda()
    plen = torch.tensor([P], dtype=torch.int32)
    out, lse = fe.fe_tree_attention(t, store, 0, q, plen.cuda(), scale=1.0)
    assert fe.fe_target_status(t) == fe.FE_OK
    check_attention(c, store, None, q, plen, torch.tensor([T]), None, out, lse, scale=1.0)
