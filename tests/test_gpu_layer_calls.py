"""Calls of the dense operators that programs may make at the edge of what include/fe_layer.h and the binding
allow."""
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
