"""How matrix products are divided, and that the sizes of test_gpu_layer_tiles.py reach every mode of the kernels."""
import ctypes
import os
import subprocess

import pytest

import gemm_shapes as shapes

HERE = os.path.dirname(os.path.abspath(__file__))
SMS, PAIRS = 152, 76
FORMS = {"gated": (1, 0, 0, 0), "plain": (0, 0, 0, 0), "grad": (0, 0, 1, 1), "columns": (0, 0, 0, 1), "rows": (0, 0, 0, 1), "twice": (0, 1, 0, 1)}


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    from paper_2509_20416_gb300 import build
    lib = str(tmp_path_factory.mktemp("plan") / "gemm_plan.so")
    subprocess.run([build.nvcc(), *build.ARCH, *build.NVCC_FLAGS, "-shared", os.path.join(HERE, "cuda", "gemm_plan.cu"), "-o", lib],
                   check=True, capture_output=True, text=True)
    lib = ctypes.CDLL(lib)
    i, l = ctypes.c_int, ctypes.c_int64
    lib.gemm_tc_plan.argtypes = [l] + [i] * 6 + [ctypes.POINTER(l)]
    lib.gemm_few_plan.argtypes = [l] + [i] * 4 + [ctypes.POINTER(l)]
    lib.gemm_simt_large.argtypes = [l] + [i] * 4
    return lib


def tc(plan, form, M, N):
    out = (ctypes.c_int64 * 4)()
    plan.gemm_tc_plan(M, N, *FORMS[form], SMS, out)
    return list(out)


def few(plan, M, N, K, gated):
    out = (ctypes.c_int64 * 3)()
    plan.gemm_few_plan(M, N, K, gated, SMS, out)
    return list(out)


# the widths that a form takes with three tiles or more of a pair, and with two
MANY = {"gated": {160, 192, 224, 256}, "plain": {160, 192, 224, 256}, "grad": {224, 256}, "columns": {224, 256}, "rows": {224, 256}, "twice": {224, 256}}
TWO = {f: w | {128} for f, w in MANY.items()}


def test_sizes_reach_every_form_and_width(plan):
    two, many = set(), set()
    for s in shapes.BLOCKS:
        for form, M, N, K in shapes.products(*s):
            width, tiles, stages, _ = tc(plan, form, M, N)
            slices = -(-K // 64)
            if tiles > PAIRS and slices > 2 * stages:
                two.add((form, width))
            if tiles > 2 * PAIRS and slices > stages + 1:  # a third tile: an accumulator's second use, behind the wait for it
                many.add((form, width))
    assert two >= {(f, w) for f, ws in TWO.items() for w in ws}
    assert many >= {(f, w) for f, ws in MANY.items() for w in ws}
    widths = {tc(plan, "plain", M, N)[0] for M, _, N in shapes.PROJECTS}
    assert len(widths) >= 3 and all(tc(plan, "plain", M, N)[1] > PAIRS for M, _, N in shapes.PROJECTS)
    for s in shapes.ODD_BLOCKS:
        assert all(tc(plan, form, M, N)[1] > 1 for form, M, N, _ in shapes.products(*s))


def test_no_other_width_is_taken(plan):
    """Over a wide range of sizes no form with three tiles a pair takes a width that the sizes above leave out."""
    for form, widths in MANY.items():
        seen = set()
        for M in range(129, 9000, 211):
            for N in range(8, 16000, 317):
                width, tiles, stages, bytes_ = tc(plan, form, M, N)
                assert stages >= 4 and bytes_ <= (192 - 64 * (form == "grad")) * 1024
                if tiles > 2 * PAIRS:
                    seen.add(width)
        assert seen <= widths, form


def test_sizes_turn_the_rings_of_few_rows(plan):
    for gated, sizes in ((0, shapes.FEW), (1, shapes.FEW_GATED)):
        ranks = set()
        for M, K, N in sizes:
            r, stages, smem = few(plan, M, N, K, gated)
            assert -(-K // 64) // r >= 3 * stages, (M, K, N)
            assert smem <= 224 * 1024
            ranks.add(r)
        assert len(ranks) >= 3


def test_few_rows_never_ask_for_more_tensor_memory_than_an_sm_has(plan):
    """A cluster's CTAs wait for one another, so those that fit an SM at once must not wait for tensor memory that
    another cluster holds: shared memory bounds them before the 512 columns do."""
    for gated in (0, 1):
        for M in range(1, 129):
            cols = 32
            while cols < -(-M // 16) * 16:
                cols *= 2
            for K in (1, 64, 65, 128, 129, 200, 512, 1000, 4096, 20000):
                for N in (1, 600, 5000, 9728, 19456, 19457, 29184, 30000, 60000, 200000, 1 << 24):
                    smem = few(plan, M, N, K, gated)[2] + 1024  # (what the system takes of each CTA's)
                    assert (228 * 1024 // smem) * cols <= 512, (M, K, N)


def test_sizes_reach_large_float32_tiles(plan):
    reached = set()
    for s in shapes.BLOCKS + shapes.ODD_BLOCKS:
        for form, M, N, _ in shapes.products(*s):
            if plan.gemm_simt_large(M, N, int(form == "gated"), int(form == "twice"), SMS):
                reached.add((form, N % 4 == 0))
    assert reached == {(f, a) for f in FORMS for a in (True, False)}
