"""Python binding of the dense operators of a target layer (include/fe_layer.h): matrix products
with bias, activation and residual, the gated feed-forward block, the norms around a block, and the
log probabilities of given tokens, on a handle of fe_target_init.

As the rest of the package, these functions only marshal arguments. Tensors are CUDA tensors of the
handle's type (fe_token_logprobs: float32 or bfloat16 logits, whatever the handle's), [..., columns]
with contiguous columns and rows one stride apart, such as column slices of a fused projection.
`stream` (a torch stream or a raw handle) is where a call runs, the current stream unless given;
ordering it with others is the caller's. Where autograd records and neither outputs nor a stream
are given, the results are differentiable (once); outputs given carry no graph, and count as changed in
place. The _backward functions are the same gradients as plain calls, for a captured step or a training
loop of one's own. (PyTorch's engine joins the streams of a leaf's graphs: a backward pass is captured
while no eager graph of the same leaves lives, or with the _backward functions.) Workspaces are
allocated for each call, so that calls and captured graphs do not share them.
"""
from __future__ import annotations

import ctypes
import struct

import torch
from torch.autograd.function import once_differentiable

from . import _check, _lib, _stream, _vp, FE_BF16, FE_F32
from .target import Target, _empty, _raw_stream, _side, _written

_ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
_M = "Pq"  # fe_mat
_ARGS = {
    "fe_project": "qii" + 2 * _M + "P" + 3 * _M + "i4xPq",
    "fe_project_backward": "qii" + 6 * _M + "Pi4xPq",
    "fe_gated_ffn": "qii" + 6 * _M + "i4xPq",
    "fe_gated_ffn_backward": "qiii4x" + 11 * _M + "i4xPq",
    "fe_block_norm": "qii" + 3 * _M + "qPPfff4x" + 2 * _M,
    "fe_block_norm_backward": "qii" + 3 * _M + "qPPfff4x" + 5 * _M + "PPPq",
    "fe_token_logprobs": "qiii4x" + _M + "if" + 7 * "P",
    "fe_token_logprobs_backward": "qiii4x" + _M + "if" + 8 * "P" + _M,
}
_PACK = {name: struct.Struct("@" + fmt).pack for name, fmt in _ARGS.items()}
_CALL, _WORK = {}, {}
for _name in _ARGS:
    _f = _CALL[_name] = getattr(_lib, _name)
    _f.argtypes = [_vp, ctypes.c_char_p, _vp]
    _f.restype = ctypes.c_int
    if hasattr(_lib, _name + "_work"):
        _f = _WORK[_name] = getattr(_lib, _name + "_work")
        _f.argtypes = [_vp, ctypes.c_char_p]
        _f.restype = ctypes.c_int64
_NONE = (0, 0)


def _mat(x, dtype, shape) -> tuple:
    """The address and row stride of [..., columns] as a matrix; (0, 0) for None."""
    if x is None:
        return _NONE
    if x.dtype != dtype or x.shape != shape or not x.is_cuda:
        _wrong(x, dtype, shape)
    if x.is_contiguous():
        n = shape[-1]
        return x.data_ptr(), n if x.numel() > n else 0
    row = _row(x)
    if row is None:
        raise ValueError(f"columns must be contiguous and rows one stride apart, got strides {tuple(x.stride())} of {tuple(x.shape)}")
    return x.data_ptr(), row


def _wrong(x, dtype, shape) -> None:
    if not x.is_cuda:
        raise ValueError("buffers the kernels access must be CUDA tensors")
    raise ValueError(f"expected a {dtype} tensor of shape {tuple(shape)}, got {x.dtype} {tuple(x.shape)}")


def _row(x):
    """The row stride of [..., columns], 0 for one row; None where there is no single one."""
    shape, strides = x.shape, x.stride()
    if shape[-1] != 1 and strides[-1] != 1:
        return None
    row = span = None
    for n, s in zip(shape[-2::-1], strides[-2::-1]):
        if n == 1:
            continue
        if row is None:
            row = s
        elif s != span:
            return None
        span = n * s
    return row or 0


def _dense(x):
    """x, copied where it has no single row stride (gradients may come in any layout)."""
    return x if x.is_contiguous() or _row(x) is not None else x.contiguous()


def _vec(x, dtype, n) -> int:
    """The address of a contiguous vector of n elements (0 for None)."""
    if x is None:
        return 0
    if x.dtype != dtype or x.shape != (n,) or not x.is_contiguous() or not x.is_cuda:
        if not x.is_cuda:
            raise ValueError("buffers the kernels access must be CUDA tensors")
        raise ValueError(f"expected a contiguous {dtype} tensor of {n} elements, got {x.dtype} {tuple(x.shape)}")
    return x.data_ptr()


def _rows_of(x) -> int:
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError(f"expected rows of at least one element, got {tuple(x.shape)}")
    return x.numel() // x.shape[-1]


def _new(shape, like, side, dtype=None):
    """A new output of a call (on `side`: allocated there). (torch.empty: half the time of Tensor.new_empty.)"""
    if side is None:
        return torch.empty(shape, dtype=like.dtype if dtype is None else dtype, device=like.device)
    return _empty(shape, like.dtype if dtype is None else dtype, like.device, side)


def _out(x, shape, like, side):
    return _new(shape, like, side) if x is None else x


def _act(act: str) -> int:
    if act not in _ACTS:
        raise ValueError(f"act must be one of {sorted(_ACTS)}, got {act!r}")
    return _ACTS[act]


def _call(name: str, t: Target, side, tensors: tuple, args: tuple) -> None:
    """Pack the arguments (without the workspace) and call the library on the current stream or on `side`; the
    given `tensors` must lie on the current device."""
    dev = torch.cuda.current_device()
    like = None
    for x in tensors:
        if x is not None:
            like = x
            if x.get_device() != dev:
                raise ValueError("buffers the kernels access must be on the current device")
            if side is not None:
                x.record_stream(side)
    raw = side.cuda_stream if side is not None else _raw_stream(dev) if _raw_stream is not None else _stream(None)
    pack, size = _PACK[name], _WORK.get(name)
    if size is not None:
        packed = pack(*args, 0, 0)
        need = size(t.ptr, packed)
        if need > 0:
            work = _new((need,), like, side, torch.uint8)
            packed = pack(*args, work.data_ptr(), need)
    else:
        packed = pack(*args)
    code = _CALL[name](t.ptr, packed, raw)
    if code:
        _check(code, name)


def _recorded(stream) -> bool:
    """Whether a call without outputs given takes part in autograd, if an input does."""
    return torch.is_grad_enabled() and _side(stream) is None


def _wants(*inputs) -> bool:
    for x in inputs:
        if x is not None and x.requires_grad:
            return True
    return False


def _shaped(x, n: int) -> torch.Size:
    return x.shape if x.shape[-1] == n else x.shape[:-1] + (n,)


# ---- fe_project ---------------------------------------------------------------------------


def fe_project(t: Target, x, w, bias=None, act: str = "none", residual=None, out=None, pre=None, stream=None):
    """act(x w^T + bias) + residual (include/fe_layer.h): x [..., K], w [N, K], bias [N], residual
    [..., N]; act: "none", "relu", "silu" or "gelu". out may be the residual itself; pre [..., N], float32,
    takes x w^T + bias, for fe_project_backward."""
    if out is None and pre is None and _recorded(stream) and _wants(x, w, bias, residual):
        return _Project.apply(t, act, x, w, bias, residual)
    N, K = w.shape
    side, shape, M = _side(stream), _shaped(x, N), _rows_of(x)
    args = (M, N, K, *_mat(x, t.dtype, _shaped(x, K)), *_mat(w, t.dtype, (N, K)), _vec(bias, t.dtype, N),
            *_mat(residual, t.dtype, shape))
    given = out, pre
    out = _out(out, shape, x, side)
    args += (*_mat(out, t.dtype, shape), *_mat(pre, torch.float32, shape), _act(act))
    if M:
        _call("fe_project", t, side, (x, w, bias, residual, out, pre), args)
    _written(*given)
    return out


def fe_project_backward(t: Target, dout, x=None, w=None, pre=None, act: str = "none", dx: bool = True, dw: bool = True,
                        dbias: bool = False, stream=None) -> tuple:
    """Gradients (dx, dw, dbias) of fe_project for dout [..., N], None for those not asked for (the
    residual's is dout). w is needed for dx, x for dw, pre for an activation."""
    if (dx and w is None) or (dw and x is None) or (act != "none" and pre is None):
        raise ValueError("dx needs w, dw needs x, and an activation needs pre")
    N, M = dout.shape[-1], _rows_of(dout)
    K = w.shape[1] if w is not None else x.shape[-1] if x is not None else 1
    side, like = _side(stream), dout
    gx = _out(None, _shaped(dout, K), like, side) if dx else None
    gw = _out(None, (N, K), like, side) if dw else None
    gb = _out(None, (N,), like, side) if dbias else None
    args = (M, N, K, *_mat(x if dw else None, t.dtype, _shaped(dout, K)), *_mat(w if dx else None, t.dtype, (N, K)),
            *_mat(dout, t.dtype, _shaped(dout, N)), *_mat(pre, torch.float32, dout.shape), *_mat(gx, t.dtype, _shaped(dout, K)),
            *_mat(gw, t.dtype, (N, K)), _vec(gb, t.dtype, N), _act(act))
    if M and (dx or dw or dbias):
        _call("fe_project_backward", t, side, (dout, x, w, pre, gx, gw, gb), args)
    elif not M:
        _zero(side, gw, gb)
    return gx, gw, gb


def _zero(side, *tensors) -> None:
    """Gradients of a call without rows."""
    with torch.cuda.stream(side):
        for x in tensors:
            if x is not None:
                x.zero_()


class _Project(torch.autograd.Function):
    @staticmethod
    def forward(ctx, t, act, x, w, bias, residual):
        need = any(ctx.needs_input_grad[2:5])
        pre = _new(_shaped(x, w.shape[0]), x, None, torch.float32) if need and act != "none" else None
        out = fe_project(t, x, w, bias, act, residual, pre=pre)
        ctx.t, ctx.act = t, act
        ctx.save_for_backward(x if ctx.needs_input_grad[3] else None, w if ctx.needs_input_grad[2] else None, pre)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        x, w, pre = ctx.saved_tensors
        _, _, nx, nw, nb, nr = ctx.needs_input_grad
        g = (None, None, None)
        if nx or nw or nb:
            g = fe_project_backward(ctx.t, _dense(dout), x, w, pre, ctx.act, nx, nw, nb)
        return None, None, *g, dout if nr else None


# ---- fe_gated_ffn --------------------------------------------------------------------------


def fe_gated_ffn(t: Target, x, w_gate, w_up, w_down=None, act: str = "silu", residual=None, out=None, gate_pre=None,
                 up_pre=None, stream=None):
    """A gated feed-forward block (include/fe_layer.h): h = act(x w_gate^T) * (x w_up^T) for x [..., K] and
    w_gate, w_up [F, K]; with w_down [N, F] the whole block, h w_down^T + residual (fe_project). gate_pre
    and up_pre [..., F], float32, take the two products, for fe_gated_ffn_backward."""
    if w_down is None and residual is not None:
        raise ValueError("a residual needs w_down")
    if out is None and gate_pre is None and up_pre is None and _recorded(stream) and _wants(x, w_gate, w_up, w_down, residual):
        return _Gated.apply(t, act, x, w_gate, w_up, w_down, residual)
    if w_down is not None:
        with torch.no_grad():  # (not recorded as a whole: neither of its parts is)
            h = fe_gated_ffn(t, x, w_gate, w_up, act=act, gate_pre=gate_pre, up_pre=up_pre, stream=stream)
            return fe_project(t, h, w_down, residual=residual, out=out, stream=stream)
    F, K = w_gate.shape
    side, shape, M = _side(stream), _shaped(x, F), _rows_of(x)
    args = (M, F, K, *_mat(x, t.dtype, _shaped(x, K)), *_mat(w_gate, t.dtype, (F, K)), *_mat(w_up, t.dtype, (F, K)))
    given = out, gate_pre, up_pre
    out = _out(out, shape, x, side)
    args += (*_mat(out, t.dtype, shape), *_mat(gate_pre, torch.float32, shape), *_mat(up_pre, torch.float32, shape), _act(act))
    if M:
        _call("fe_gated_ffn", t, side, (x, w_gate, w_up, out, gate_pre, up_pre), args)
    _written(*given)
    return out


def fe_gated_ffn_backward(t: Target, dout, gate_pre, up_pre, x=None, w_gate=None, w_up=None, w_down=None, act: str = "silu",
                          dx: bool = True, dw: bool = True, dw_down: bool | None = None, stream=None) -> tuple:
    """Gradients (dx, dw_gate, dw_up, dw_down) of fe_gated_ffn for dout, [..., F] or with w_down [..., N], None for
    those not asked for (dw_down: by default with w_down). w_gate and w_up are needed for dx, x for dw."""
    dw_down = w_down is not None if dw_down is None else dw_down
    if (dx and (w_gate is None or w_up is None)) or (dw and x is None) or (dw_down and w_down is None):
        raise ValueError("dx needs w_gate and w_up, dw needs x, dw_down needs w_down")
    if not (dx or dw or dw_down):
        return None, None, None, None
    F, M, N = gate_pre.shape[-1], _rows_of(dout), dout.shape[-1]
    K = w_gate.shape[1] if dx else x.shape[-1] if dw else 1
    side, shape = _side(stream), _shaped(dout, F)
    gx = _out(None, _shaped(dout, K), dout, side) if dx else None
    gg, gu = (_out(None, (F, K), dout, side) if dw else None for _ in range(2))
    gd = _out(None, (N, F), dout, side) if dw_down else None
    args = (M, F, K, N, *_mat(x if dw else None, t.dtype, _shaped(dout, K)), *_mat(w_gate if dx else None, t.dtype, (F, K)),
            *_mat(w_up if dx else None, t.dtype, (F, K)), *_mat(w_down, t.dtype, (N, F)),
            *_mat(dout, t.dtype, shape if w_down is None else dout.shape), *_mat(gate_pre, torch.float32, shape),
            *_mat(up_pre, torch.float32, shape), *_mat(gx, t.dtype, _shaped(dout, K)), *_mat(gg, t.dtype, (F, K)),
            *_mat(gu, t.dtype, (F, K)), *_mat(gd, t.dtype, (N, F)), _act(act))
    if M:
        _call("fe_gated_ffn_backward", t, side, (dout, x, w_gate, w_up, w_down, gate_pre, up_pre, gx, gg, gu, gd), args)
    else:
        _zero(side, gg, gu, gd)
    return gx, gg, gu, gd


class _Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, t, act, x, w_gate, w_up, w_down, residual):
        g, u = (_new(_shaped(x, w_gate.shape[0]), x, None, torch.float32) for _ in range(2))
        ctx.t, ctx.act = t, act
        _, _, nx, ng, nu, _, _ = ctx.needs_input_grad
        ctx.save_for_backward(g, u, x if ng or nu else None, w_gate if nx else None, w_up if nx else None, w_down)
        return fe_gated_ffn(t, x, w_gate, w_up, w_down, act, residual, gate_pre=g, up_pre=u)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        g, u, x, w_gate, w_up, w_down = ctx.saved_tensors
        _, _, nx, ng, nu, nd, nr = ctx.needs_input_grad
        gx, gg, gu, gd = fe_gated_ffn_backward(ctx.t, _dense(dout), g, u, x, w_gate, w_up, w_down, ctx.act, nx, ng or nu, nd)
        return None, None, gx, gg if ng else None, gu if nu else None, gd, dout if nr else None


# ---- fe_block_norm --------------------------------------------------------------------------


def fe_block_norm(t: Target, x, z=None, post: bool | None = None, post_weight=None, gate=None, gate_rows: int | None = None,
                  scale: float = 1.0, pre_weight=None, offset: float = 0.0, eps: float = 1e-5, y=None, n=None, pre: bool = True,
                  stream=None) -> tuple:
    """The norms around a block (include/fe_layer.h): y = x + scale gate p with p the block's output z
    [..., d], normed if post (the default where post_weight is given), and n = norm(y), which the next
    block takes. gate is [groups, d] for groups of gate_rows rows (default: rows / groups, rounded up),
    or [d] for all. Without z, y is x (returned as it is unless an output is given). Returns (y, n), n None
    if not pre; outputs given may be z, or y x, themselves."""
    post = post_weight is not None if post is None else post
    if post_weight is not None and not post:
        raise ValueError("post_weight without post")
    if z is None and (post or gate is not None):
        raise ValueError("a norm or a gate of the block's output needs z")
    if not pre and (pre_weight is not None or n is not None or (z is None and y is None)):
        raise ValueError("without a norm before the next block there is no pre_weight or n, and z or y is needed")
    if gate is not None and gate.dim() == 1:
        gate = gate[None]
    R, shape = _rows_of(x), x.shape
    gate_rows = _gate_rows(gate, gate_rows, R)
    opts = (bool(post), gate_rows, float(scale), float(offset), float(eps))
    if y is None and n is None and _recorded(stream) and _wants(x, z, post_weight, gate, pre_weight):
        out = _BlockNorm.apply(t, opts, pre, x, z, post_weight, gate, pre_weight)
        return (x, out) if z is None else out if pre else (out, None)
    side, given = _side(stream), (y, n)
    y = None if y is None and z is None else _out(y, shape, x, side)
    n = _out(n, shape, x, side) if pre else None
    args = _norm_args(t, opts, x, z, post_weight, gate, pre_weight) + (*_mat(y, t.dtype, shape), *_mat(n, t.dtype, shape))
    if R:
        _call("fe_block_norm", t, side, (x, z, post_weight, gate, pre_weight, y, n), args)
    _written(*given)
    return x if y is None else y, n


def _gate_rows(gate, rows, R: int) -> int:
    if gate is None:
        return 0
    if gate.dim() != 2:
        raise ValueError("gate must be [groups, d] or [d]")
    if rows is None:
        rows = -(-R // max(gate.shape[0], 1))
    if rows < 1 and R:
        raise ValueError("gate_rows must be positive")
    if R and gate.shape[0] != -(-R // rows):
        raise ValueError(f"gate has {gate.shape[0]} rows, {R} rows in groups of {rows} need {-(-R // rows)}")
    return rows


def _norm_args(t, opts, x, z, post_weight, gate, pre_weight) -> tuple:
    post, rows, scale, offset, eps = opts
    shape, dtype = x.shape, t.dtype
    d = shape[-1]
    return (_rows_of(x), d, int(post), *_mat(x, dtype, shape), *_mat(z, dtype, shape),
            *_mat(gate, dtype, None if gate is None else (gate.shape[0], d)), rows, _vec(post_weight, dtype, d),
            _vec(pre_weight, dtype, d), scale, offset, eps)


def fe_block_norm_backward(t: Target, x, z=None, post: bool | None = None, post_weight=None, gate=None, gate_rows: int | None = None,
                           scale: float = 1.0, pre_weight=None, offset: float = 0.0, eps: float = 1e-5, dy=None, dn=None,
                           need=(True, True, True, True, True), stream=None) -> tuple:
    """Gradients (dx, dz, dpost_weight, dgate, dpre_weight) of fe_block_norm for dy and dn (either may be
    None), None for those that `need` leaves out or whose input is not given."""
    post = post_weight is not None if post is None else post
    if gate is not None and gate.dim() == 1:
        dx, dz, dp, dg, dw = fe_block_norm_backward(t, x, z, post, post_weight, gate[None], gate_rows, scale, pre_weight, offset, eps,
                                                    dy, dn, need, stream)
        return dx, dz, dp, None if dg is None else dg[0], dw
    if dy is None and dn is None:
        raise ValueError("a gradient of y or n is needed")
    R, d = _rows_of(x), x.shape[-1]
    opts = (bool(post), _gate_rows(gate, gate_rows, R), float(scale), float(offset), float(eps))
    side = _side(stream)
    shapes = (x.shape, x.shape, (d,), None if gate is None else tuple(gate.shape), (d,))
    dx, dz, dp, dg, dw = (_out(None, s, x, side) if w and i is not None else None
                          for i, w, s in zip((x, z, post_weight, gate, pre_weight), need, shapes))
    if all(g is None for g in (dx, dz, dp, dg, dw)):
        return None, None, None, None, None
    args = _norm_args(t, opts, x, z, post_weight, gate, pre_weight) + \
        (*_mat(dy, t.dtype, x.shape), *_mat(dn, t.dtype, x.shape), *_mat(dx, t.dtype, x.shape), *_mat(dz, t.dtype, x.shape),
         *_mat(dg, t.dtype, shapes[3]), _vec(dp, t.dtype, d), _vec(dw, t.dtype, d))
    if R:
        _call("fe_block_norm_backward", t, side, (x, z, post_weight, gate, pre_weight, dy, dn, dx, dz, dp, dg, dw), args)
    else:
        _zero(side, dp, dg, dw)
    return dx, dz, dp, dg, dw


class _BlockNorm(torch.autograd.Function):
    """(y, n), or the one of them that is wanted: without z y is x, without pre there is no n."""

    @staticmethod
    def forward(ctx, t, opts, pre, x, z, post_weight, gate, pre_weight):
        ctx.t, ctx.opts, ctx.pre = t, opts, pre
        ctx.save_for_backward(x, z, post_weight, gate, pre_weight)
        ctx.set_materialize_grads(False)
        post, rows, scale, offset, eps = opts
        y, n = fe_block_norm(t, x, z, post, post_weight, gate, rows, scale, pre_weight, offset, eps, pre=pre)
        return n if z is None else (y, n) if pre else y

    @staticmethod
    @once_differentiable
    def backward(ctx, *grads):
        if all(g is None for g in grads):
            return (None,) * 8
        x, z, post_weight, gate, pre_weight = ctx.saved_tensors
        post, rows, scale, offset, eps = ctx.opts
        grads = tuple(None if g is None else _dense(g) for g in grads)
        dy, dn = grads if len(grads) == 2 else (None, *grads) if z is None else (*grads, None)
        return None, None, None, *fe_block_norm_backward(ctx.t, x, z, post, post_weight, gate, rows, scale, pre_weight, offset, eps, dy,
                                                         dn, ctx.needs_input_grad[3:])


# ---- fe_token_logprobs -----------------------------------------------------------------------

_LOGITS = {torch.float32: FE_F32, torch.bfloat16: FE_BF16}


def _contiguous(x, side):
    """x, copied on the call's stream where it is not contiguous; there x is in use until the copy has run."""
    if x.is_contiguous() or side is None:
        return x.contiguous()
    x.record_stream(side)
    with torch.cuda.stream(side):
        return x.contiguous()


def _tokens(x, lead, side) -> tuple:
    """tokens [..., J] or [...] (one a row) as [..., J], and J."""
    if x is None:
        return None, 0
    if not x.is_cuda:
        raise ValueError("buffers the kernels access must be CUDA tensors")
    x = x[..., None] if x.shape == lead else x
    if x.dtype != torch.int32 or x.shape[:-1] != lead:
        raise ValueError(f"tokens must be int32 of shape {tuple(lead)} or {tuple(lead)} + (J,), got {x.dtype} {tuple(x.shape)}")
    return _contiguous(x, side), x.shape[-1]


def fe_token_logprobs(t: Target, logits, tokens=None, top: int = 0, temperature: float = 1.0, stats=None, stream=None) -> tuple:
    """Log probabilities under softmax(logits / temperature) (include/fe_layer.h): logits [..., V] float32
    or bfloat16, tokens int32 [..., J] or [...] (negative: none). Returns float32 (logprob, as tokens;
    entropy [...]; lse [...]; top_id [..., top] int32; top_logprob [..., top]): the `top` most probable
    tokens, in order. logprob is None without tokens. stats [..., 2] takes what fe_token_logprobs_backward
    needs of a row."""
    if stats is None and _recorded(stream) and logits.requires_grad:
        out = _Logprobs.apply(t, logits, tokens, top, temperature)
        return (None, *out[1:]) if tokens is None else out
    lead, V, side, f32 = logits.shape[:-1], logits.shape[-1], _side(stream), torch.float32
    tok, J = _tokens(tokens, lead, side)
    if logits.dtype not in _LOGITS:
        raise ValueError(f"logits must be float32 or bfloat16, got {logits.dtype}")
    logprob = None if tokens is None else _new(tokens.shape, logits, side, f32)
    entropy, lse = _new(lead, logits, side, f32), _new(lead, logits, side, f32)
    ids, lps = _new(lead + (top,), logits, side, torch.int32), _new(lead + (top,), logits, side, f32)
    if stats is not None and (stats.dtype != torch.float32 or stats.shape != lead + (2,) or not stats.is_contiguous() or not stats.is_cuda):
        raise ValueError(f"stats must be a contiguous float32 CUDA tensor of shape {tuple(lead) + (2,)}")
    p = lambda x: 0 if x is None else x.data_ptr()
    R = _rows_of(logits)
    args = (R, V, J, top, *_mat(logits, logits.dtype, logits.shape), _LOGITS[logits.dtype], float(temperature), p(tok), p(logprob),
            p(entropy), p(lse), p(stats), p(ids), p(lps))
    if R:
        _call("fe_token_logprobs", t, side, (logits, tok, logprob, entropy, lse, stats, ids, lps), args)
    _written(stats)
    return logprob, entropy, lse, ids, lps


def fe_token_logprobs_backward(t: Target, logits, stats, tokens=None, dlogprob=None, entropy=None, dentropy=None, dlse=None, top_id=None,
                               dtop_logprob=None, temperature: float = 1.0, dlogits=None, stream=None):
    """dlogits [..., V] of fe_token_logprobs, for the gradients of its results (None: zero); stats, entropy
    and top_id are the forward call's. dlogits may be the logits themselves."""
    lead, V, side = logits.shape[:-1], logits.shape[-1], _side(stream)
    tok, J = _tokens(tokens, lead, side)
    if logits.dtype not in _LOGITS:
        raise ValueError(f"logits must be float32 or bfloat16, got {logits.dtype}")
    if (dlogprob is not None and tok is None) or (dentropy is not None and entropy is None) or \
            (dtop_logprob is not None and top_id is None):
        raise ValueError("dlogprob needs tokens, dentropy needs entropy, and dtop_logprob needs top_id")

    def flat(x, shape, dtype=torch.float32):
        if x is None:
            return None
        if not x.is_cuda:
            raise ValueError("buffers the kernels access must be CUDA tensors")
        if x.dtype != dtype or x.shape != shape:
            raise ValueError(f"expected {dtype} of shape {tuple(shape)}, got {x.dtype} {tuple(x.shape)}")
        return _contiguous(x, side)

    K = 0 if top_id is None else top_id.shape[-1]
    given = (flat(stats, lead + (2,)), flat(entropy, lead), flat(dlogprob, None if tokens is None else tokens.shape), flat(dentropy, lead),
             flat(dlse, lead), flat(dtop_logprob, lead + (K,)))
    top_id = flat(top_id, lead + (K,), torch.int32)
    out = dlogits
    dlogits = _out(dlogits, logits.shape, logits, side)
    p = lambda x: 0 if x is None else x.data_ptr()
    R = _rows_of(logits)
    args = (R, V, J, K, *_mat(logits, logits.dtype, logits.shape), _LOGITS[logits.dtype], float(temperature), p(tok), p(top_id),
            *(p(x) for x in given), *_mat(dlogits, logits.dtype, logits.shape))
    if R:
        _call("fe_token_logprobs_backward", t, side, (logits, tok, top_id, *given, dlogits), args)
    _written(out)
    return dlogits


class _Logprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, t, logits, tokens, top, temperature):
        stats = _new(logits.shape[:-1] + (2,), logits, None, torch.float32)
        out = fe_token_logprobs(t, logits, tokens, top, temperature, stats)
        logprob, entropy, _, ids, _ = out
        ctx.t, ctx.temperature = t, temperature
        ctx.save_for_backward(logits, tokens, entropy, stats, ids)
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(ids)
        return (logits.new_empty(0, dtype=torch.float32) if logprob is None else logprob, *out[1:])

    @staticmethod
    @once_differentiable
    def backward(ctx, dlogprob, dentropy, dlse, _, dtop):
        if all(g is None for g in (dlogprob, dentropy, dlse, dtop)):
            return None, None, None, None, None
        logits, tokens, entropy, stats, ids = ctx.saved_tensors
        g = fe_token_logprobs_backward(ctx.t, logits, stats, tokens, None if tokens is None else dlogprob, entropy, dentropy, dlse, ids,
                                       dtop, ctx.temperature)
        return None, g, None, None, None
