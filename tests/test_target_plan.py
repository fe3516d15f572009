"""The attention's schedule counts units of work in 32 bits: a shape whose calls could need more is
refused, for every type by the constants that its own kernel counts with."""
import ctypes
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
F32, BF16, E4M3 = 0, 1, 2


@pytest.fixture(scope="module")
def fits(tmp_path_factory):
    from paper_2509_20416_gb300 import build
    lib = str(tmp_path_factory.mktemp("plan") / "plan_fits.so")
    subprocess.run([build.nvcc(), *build.ARCH, *build.NVCC_FLAGS, "-shared", os.path.join(HERE, "cuda", "plan_fits.cu"),
                    "-o", lib], check=True, capture_output=True, text=True)
    f = ctypes.CDLL(lib).plan_fits
    f.argtypes = [ctypes.c_int] * 7
    return f


def units(dtype, cache, B, Hkv, G, T, P):
    """The length of the line of units of a masked call: B sequences of T nodes behind P slots. An
    item costs its start, one or two units a tile, and over bfloat16 one more for a tile with nodes
    where it costs two."""
    ROWS, TN = (64, 64) if dtype == F32 else (256, 128)
    over, tail = {F32: (1, 0), BF16: (4, 1), E4M3: (6, 0)}[dtype if dtype == F32 else cache]
    rows = T * G
    nb, nt = -(-rows // ROWS), -(-(P + T) // TN)
    extra = tail * max(nt - P // TN, 0)
    w = [1 if dtype == F32 or rows - m * ROWS <= 128 else 2 for m in (0, nb - 1)]
    item = lambda w: over + w * nt + (w - 1) * extra
    return B * Hkv * ((nb - 1) * item(w[0]) + item(w[1]))


CASES = [(dtype, cache, B, Hkv, G, seq) for dtype, cache in ((F32, F32), (BF16, BF16), (BF16, E4M3))
         for B, Hkv, G, seq in ((1, 1, 128, 1 << 20), (1, 8, 8, 1 << 20), (4, 1, 16, 1 << 22), (32, 2, 3, 1 << 17), (7, 40, 1, 1 << 16))]


@pytest.mark.parametrize("dtype,cache,B,Hkv,G,seq", CASES)
def test_no_call_of_an_accepted_shape_overflows(fits, dtype, cache, B, Hkv, G, seq):
    """T is raised to the most that is accepted; the longest calls of that T, without a prefix and with
    the longest one, stay below 2^31. The guard is no tighter than a factor of three."""
    lo, hi = 1, seq
    while lo < hi:
        mid = (lo + hi + 1) // 2
        lo, hi = (mid, hi) if fits(dtype, cache, B, Hkv, mid, G, seq) else (lo, mid - 1)
    for T in (lo, max(1, lo - 1), lo // 2 + 1):
        for P in (0, 1, (seq - T) // 2, seq - T):
            assert units(dtype, cache, B, Hkv, G, T, P) < 2**31, (T, P)
    if lo < seq:
        assert 3 * units(dtype, cache, B, Hkv, G, lo + 1, seq - lo - 1) >= 2**31


def test_trees_of_half_a_million_nodes_over_bfloat16(fits):
    """128 heads on one KV head, no prefix, a mask over 440 thousand nodes: more than 2^31 units over
    bfloat16, fewer over e4m3."""
    T = 440000
    assert units(BF16, BF16, 1, 1, 128, T, 0) >= 2**31 > units(BF16, E4M3, 1, 1, 128, T, 0)
    assert not fits(BF16, BF16, 1, 1, T, 128, T)
    assert fits(BF16, E4M3, 1, 1, T, 128, T)
