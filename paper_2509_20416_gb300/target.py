"""Python binding of the target-side operators (include/fe_target.h): rotary positions, the
key/value cache's write, read and accepted-row moves, and attention of a draft tree over it.

As the rest of the package, these functions only marshal arguments. Row tensors (queries,
keys, values, outputs) are CUDA tensors [B, T, heads, head_dim] of the handle's type with any
strides whose innermost dimension is contiguous, such as views of a fused projection; integer
inputs are contiguous CUDA int32 tensors. `stream` (a torch stream or a raw handle) is where a call
runs, the current stream unless given; ordering it with others is the caller's. fe_rope takes part
in autograd; the results of the cache and the attention over it, which serve, carry no graph.
"""
from __future__ import annotations

import ctypes
import math
import struct

import torch

from . import _check, _i32, _lib, _stream, _vp, FE_BF16, FE_F32

FE_E4M3 = 2
_DTYPES = {"f32": FE_F32, "bf16": FE_BF16, "e4m3": FE_E4M3}
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
_LAYOUTS = {"half": 0, "interleaved": 1}
_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "bands": 3, "yarn": 4}

_f32 = ctypes.c_float
_i64 = ctypes.c_int64


class fe_target_config(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("n_heads", "n_kv_heads", "head_dim", "max_batch", "max_seq", "page_size", "dtype",
                                    "cache_dtype", "rope_dim", "rope_layout", "rope_scaling")] + \
               [(n, _f32) for n in ("rope_theta", "rope_factor", "rope_low", "rope_high", "rope_orig")]


class fe_kv(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp)]


# The calls' argument structs (include/fe_target.h), packed in one step: filling ctypes structures
# field by field would cost more than a small kernel takes. rows: p and three strides; kv: k, v,
# k_scale, v_scale; pages: table, n_pages.
_ROWS, _KV, _PAGES = "Pqqq", "PPPP", "Pi4x"
_ARGS = {
    "fe_rope": "ii" + 4 * _ROWS + "Pi4x",
    "fe_cache_write": "ii" + 4 * _ROWS + "PPP" + _KV + _PAGES,
    "fe_cache_read": "iiPP" + _KV + _PAGES + 2 * _ROWS,
    "fe_tree_attention": "ii" + 2 * _ROWS + "PPPPf4x" + _KV + _PAGES,
    "fe_cache_keep": "iii4xPPPP" + _PAGES,
}
_PACK = {name: struct.Struct("@" + fmt).pack for name, fmt in _ARGS.items()}
_NONE = (0, 0, 0, 0)  # rows not given

_lib.fe_target_init.argtypes = [ctypes.POINTER(fe_target_config), _vp, ctypes.POINTER(_vp)]
_lib.fe_target_init.restype = ctypes.c_int
_lib.fe_target_free.argtypes = [_vp]
_lib.fe_target_free.restype = None
_lib.fe_target_status.argtypes = [_vp, _vp]
_lib.fe_target_status.restype = ctypes.c_int
for _name in _ARGS:
    _f = getattr(_lib, _name)
    _f.argtypes = [_vp, ctypes.c_char_p, _vp]
    _f.restype = ctypes.c_int
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else None


def make_target_config(cfg: dict) -> fe_target_config:
    hd = cfg["head_dim"]
    return fe_target_config(
        cfg["n_heads"], cfg["n_kv_heads"], hd, cfg.get("max_batch", 1), cfg["max_seq"], cfg.get("page_size", 0),
        _DTYPES[cfg["dtype"]], _DTYPES[cfg.get("cache_dtype", cfg["dtype"])], cfg.get("rope_dim", hd),
        _LAYOUTS[cfg.get("rope_layout", "half")], _SCALINGS[cfg.get("rope_scaling", "none")], cfg["rope_theta"],
        cfg.get("rope_factor", 1.0), cfg.get("rope_low", 0.0), cfg.get("rope_high", 0.0), cfg.get("rope_orig", 0.0))


class Target:
    """An initialised target-side handle (owns a fe_target*)."""

    def __init__(self, ptr: int, cfg: dict):
        self.ptr = ptr
        self.cfg = dict(cfg)
        self.H, self.Hkv, self.hd = cfg["n_heads"], cfg["n_kv_heads"], cfg["head_dim"]
        self.dtype = _TORCH[cfg["dtype"]]
        self.cache_name = cfg.get("cache_dtype", cfg["dtype"])
        self.page_size, self.max_seq, self.max_batch = cfg.get("page_size", 0), cfg["max_seq"], cfg.get("max_batch", 1)
        self.scale = 1.0 / math.sqrt(self.hd)

    def __del__(self):
        self.close()

    def close(self):
        if getattr(self, "ptr", None):
            _lib.fe_target_free(self.ptr)
            self.ptr = None


def fe_target_init(cfg: dict, stream=None) -> Target:
    """cfg: n_heads, n_kv_heads, head_dim, max_seq, dtype ("f32", "bf16"), rope_theta, and
    optionally max_batch, page_size, cache_dtype ("f32", "bf16", "e4m3"; dtype), rope_dim
    (head_dim), rope_layout ("half", "interleaved"), rope_scaling ("none", "linear", "ntk",
    "bands", "yarn") with rope_factor, rope_low, rope_high and rope_orig."""
    c = make_target_config(cfg)
    out = _vp()
    _check(_lib.fe_target_init(ctypes.byref(c), _stream(stream), ctypes.byref(out)), "fe_target_init")
    return Target(out.value, cfg)


def fe_target_free(t: Target) -> None:
    t.close()


def fe_target_status(t: Target, stream=None) -> int:
    return int(_lib.fe_target_status(t.ptr, _stream(stream)))


class Cache:
    """The caches of a target's layers: k, v [layers, ...] tensors (or lists of one tensor per
    layer) in the layout of fe_kv, with float32 scales for an e4m3 cache, and the page table
    [B, ceil(max_seq / page_size)] that they share. The tensors stay the caller's; the
    addresses are laid out once, here."""

    def __init__(self, t: Target, k, v, k_scale=None, v_scale=None, page_table=None, n_pages: int = 0):
        ps = t.page_size
        rows = (n_pages, t.Hkv, ps) if ps else (t.max_batch, t.Hkv, t.max_seq)
        types = (torch.float8_e4m3fn, torch.uint8) if t.cache_name == "e4m3" else (_TORCH[t.cache_name],)
        n = len(k)
        if n < 1 or len(v) != n:
            raise ValueError("a cache needs k and v of the same number of layers")
        scaled = t.cache_name == "e4m3"
        if scaled and (k_scale is None or v_scale is None or len(k_scale) != n or len(v_scale) != n):
            raise ValueError("an e4m3 cache needs k_scale and v_scale of every layer")
        self.kv = (fe_kv * n)()
        self.rows = []  # each layer's four addresses
        for i in range(n):
            for x in (k[i], v[i]):
                _cuda(x)
                if tuple(x.shape) != rows + (t.hd,) or x.dtype not in types or not x.is_contiguous():
                    raise ValueError(f"cache layer {i} must be a contiguous {types[0]} tensor of shape {rows + (t.hd,)}")
            s = (None, None)
            if scaled:
                for x in (k_scale[i], v_scale[i]):
                    _cuda(x)
                    if tuple(x.shape) != rows or x.dtype != torch.float32 or not x.is_contiguous():
                        raise ValueError(f"scales of cache layer {i} must be contiguous float32 of shape {rows}")
                s = (k_scale[i].data_ptr(), v_scale[i].data_ptr())
            self.rows.append((k[i].data_ptr(), v[i].data_ptr()) + tuple(x or 0 for x in s))
            self.kv[i] = fe_kv(*self.rows[-1])
        self.n_layers, self.k, self.v, self.k_scale, self.v_scale = n, k, v, k_scale, v_scale
        self.page_table, self.n_pages = page_table, n_pages
        if ps:
            if page_table is None or page_table.dim() != 2 or page_table.shape[1] != -(-t.max_seq // ps):
                raise ValueError("a paged cache needs a page table [B, ceil(max_seq / page_size)]")
            _ints(page_table, tuple(page_table.shape))
        self.pages = (page_table.data_ptr() if ps else 0, n_pages)

    def _layer(self, i: int, B: int) -> tuple:
        """Addresses of layer i's buffers and of the page table, for a call of B sequences."""
        if not 0 <= i < self.n_layers:
            raise ValueError(f"layer {i} of a cache of {self.n_layers}")
        self._fits(B)
        return self.rows[i] + self.pages

    def _fits(self, B: int) -> None:
        if self.page_table is not None and self.page_table.shape[0] < B:
            raise ValueError("the page table has fewer rows than the call has sequences")

    def tensors(self):
        for x in (self.k, self.v, self.k_scale, self.v_scale, self.page_table):
            if isinstance(x, torch.Tensor):
                yield x
            elif x is not None:
                yield from x


def alloc_cache(t: Target, n_layers: int, n_pages: int = 0, page_table=None, device="cuda") -> Cache:
    """A zeroed cache of n_layers layers (paged: n_pages pages each, addressed by page_table)."""
    rows = (n_layers,) + ((n_pages, t.Hkv, t.page_size) if t.page_size else (t.max_batch, t.Hkv, t.max_seq))
    k, v = (torch.zeros(rows + (t.hd,), dtype=_TORCH[t.cache_name], device=device) for _ in range(2))
    s = [torch.ones(rows, device=device) for _ in range(2)] if t.cache_name == "e4m3" else [None, None]
    return Cache(t, k, v, *s, page_table=page_table, n_pages=n_pages)


def _cuda(x) -> None:
    if not x.is_cuda:
        raise ValueError("buffers the kernels access must be CUDA tensors")


def _ints(x, shape) -> int:
    """The address of a contiguous CUDA int32 tensor of the given shape (0 for None)."""
    if x is None:
        return 0
    _cuda(x)
    if x.dtype != torch.int32 or x.shape != shape or not x.is_contiguous():
        raise ValueError(f"expected a contiguous int32 tensor of shape {shape}, got {x.dtype} {tuple(x.shape)}")
    return x.data_ptr()


def _rows(t: Target, x, shape) -> tuple:
    """A row tensor's address and strides."""
    _cuda(x)
    s = x.stride()
    if x.dtype != t.dtype or x.shape != shape or s[3] != 1:
        raise ValueError(f"expected {t.dtype} rows {tuple(shape)} with contiguous elements, got {x.dtype} {tuple(x.shape)} "
                         f"with strides {tuple(s)}")
    return x.data_ptr(), s[0], s[1], s[2]


def _side(stream):
    """The stream of a call as PyTorch's object; None for the current stream."""
    if stream is None:
        return None
    raw = _stream(stream)
    if raw == torch.cuda.current_stream().cuda_stream:
        return None
    if isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(raw) if raw else torch.cuda.default_stream()


def _empty(shape, dtype, device, side):
    """A new output. Memory that PyTorch's allocator hands out belongs to a stream: kernels queued
    there may still use it, and another stream must not write it yet. So an output is allocated on
    the stream that writes it, and the current one, where the caller holds it, is noted as a user."""
    if side is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(side):
        x = torch.empty(shape, dtype=dtype, device=device)
    x.record_stream(torch.cuda.current_stream())
    return x


def _call(name: str, t: Target, side, tensors, *args) -> None:
    """Pack the arguments and call the library, on the current stream or on `side`: there, the
    allocator is told that `tensors` are in use."""
    if side is None:
        raw = _raw_stream(torch.cuda.current_device()) if _raw_stream is not None else _stream(None)
    else:
        raw = side.cuda_stream
        for x in tensors():
            if x is not None:
                x.record_stream(side)
    code = getattr(_lib, name)(t.ptr, _PACK[name](*args), raw)
    if code:
        _check(code, name)


def fe_rope(t: Target, q, k, pos, backward: bool = False, q_out=None, k_out=None, stream=None) -> tuple:
    """Rotary positions (include/fe_target.h) of q [B, T, H, hd] and k [B, T, Hkv, hd] (either
    may be None) at pos [B, T]; with backward, the gradient's rotation. Returns (q_out, k_out);
    pass the inputs as outputs to rotate in place. Where autograd records, new outputs on the
    current stream are differentiable in q and k."""
    if torch.is_grad_enabled() and q_out is None and k_out is None and _side(stream) is None \
            and any(x is not None and x.requires_grad for x in (q, k)):
        return _Rotation.apply(t, pos, backward, q, k)
    B, T = pos.shape
    side = _side(stream)
    qr = kr = qo = ko = _NONE
    if q is not None:
        shape = (B, T, t.H, t.hd)
        qr = _rows(t, q, shape)
        q_out = _empty(shape, t.dtype, q.device, side) if q_out is None else q_out
        qo = _rows(t, q_out, shape)
    if k is not None:
        shape = (B, T, t.Hkv, t.hd)
        kr = _rows(t, k, shape)
        k_out = _empty(shape, t.dtype, k.device, side) if k_out is None else k_out
        ko = _rows(t, k_out, shape)
    _call("fe_rope", t, side, lambda: (q, k, q_out, k_out, pos), B, T, *qr, *kr, *qo, *ko, _ints(pos, (B, T)),
          1 if backward else 0)
    return q_out, k_out


class _Rotation(torch.autograd.Function):
    """fe_rope under autograd: a rotation's gradient is its transpose."""

    @staticmethod
    def forward(ctx, t, pos, backward, q, k):
        ctx.t, ctx.turn = t, backward
        ctx.save_for_backward(pos)
        ctx.set_materialize_grads(False)
        return fe_rope(t, q, k, pos, backward)

    @staticmethod
    def backward(ctx, dq, dk):
        dq, dk = (x if x is None or x.stride(3) == 1 else x.contiguous()
                  for x in (d if need else None for d, need in zip((dq, dk), ctx.needs_input_grad[3:])))
        if dq is None and dk is None:
            return None, None, None, None, None
        return None, None, None, *fe_rope(ctx.t, dq, dk, *ctx.saved_tensors, not ctx.turn)


def fe_cache_write(t: Target, cache: Cache, layer: int, k, v, start, n_rows=None, pos=None, q=None, q_out=None,
                   stream=None):
    """Rows k, v [B, T, Hkv, hd] into slots start[b] + i of a layer's cache, the keys rotated to
    pos [B, T] if given, quantised if the cache is; with q [B, T, H, hd] also rotates the
    queries into q_out, which is returned."""
    B, T = k.shape[:2]
    shape = (B, T, t.Hkv, t.hd)
    side = _side(stream)
    qr = qo = _NONE
    if q is not None:
        qshape = (B, T, t.H, t.hd)
        qr = _rows(t, q, qshape)
        q_out = _empty(qshape, t.dtype, q.device, side) if q_out is None else q_out
        qo = _rows(t, q_out, qshape)
    _call("fe_cache_write", t, side, lambda: (k, v, start, n_rows, pos, q, q_out, *cache.tensors()), B, T,
          *_rows(t, k, shape), *_rows(t, v, shape), *qr, *qo, _ints(pos, (B, T)), _ints(start, (B,)), _ints(n_rows, (B,)),
          *cache._layer(layer, B))
    return q_out


def fe_cache_read(t: Target, cache: Cache, layer: int, start, n_rows, L: int, k_out=None, v_out=None,
                  stream=None) -> tuple:
    """Slots start[b] .. start[b] + n_rows[b] - 1 of a layer's cache as rows k, v [B, L, Hkv, hd]
    of the handle's type; rows past n_rows[b] are zero."""
    B = start.shape[0]
    side = _side(stream)
    shape = (B, L, t.Hkv, t.hd)
    k_out = _empty(shape, t.dtype, start.device, side) if k_out is None else k_out
    v_out = _empty(shape, t.dtype, start.device, side) if v_out is None else v_out
    _call("fe_cache_read", t, side, lambda: (start, n_rows, k_out, v_out, *cache.tensors()), B, L, _ints(start, (B,)),
          _ints(n_rows, (B,)), *cache._layer(layer, B), *_rows(t, k_out, shape), *_rows(t, v_out, shape))
    return k_out, v_out


def fe_tree_attention(t: Target, cache: Cache, layer: int, q, prefix_len, mask=None, n_nodes=None,
                      scale: float | None = None, out=None, lse=None, stream=None) -> tuple:
    """Attention of q [B, T, H, hd]'s nodes over a layer's cache: every node sees the slots
    before prefix_len[b], and slot prefix_len[b] + c where mask [B, T, T] (uint8) is set, or
    c <= i without a mask (consecutive tokens, single-token decoding). scale: 1 / sqrt(hd)
    unless given. Returns (out [B, T, H, hd], lse [B, T, H] float32)."""
    B, T = q.shape[:2]
    shape = (B, T, t.H, t.hd)
    qr = _rows(t, q, shape)
    side = _side(stream)
    if out is None:
        out = _empty(shape, t.dtype, q.device, side)
    if lse is None:
        lse = _empty((B, T, t.H), torch.float32, q.device, side)
    elif lse.dtype != torch.float32 or lse.shape != (B, T, t.H) or not lse.is_contiguous() or not lse.is_cuda:
        raise ValueError(f"lse must be a contiguous float32 CUDA tensor of shape {(B, T, t.H)}")
    if mask is not None and (mask.dtype not in (torch.uint8, torch.bool) or mask.shape != (B, T, T)
                             or not mask.is_contiguous() or not mask.is_cuda):
        raise ValueError(f"mask must be a contiguous uint8 CUDA tensor of shape {(B, T, T)}")
    _call("fe_tree_attention", t, side, lambda: (q, prefix_len, n_nodes, mask, out, lse, *cache.tensors()), B, T, *qr,
          *_rows(t, out, shape), lse.data_ptr(), _ints(prefix_len, (B,)), _ints(n_nodes, (B,)),
          0 if mask is None else mask.data_ptr(), t.scale if scale is None else float(scale), *cache._layer(layer, B))
    return out, lse


def fe_cache_keep(t: Target, cache: Cache, path, n_accept, start, stream=None) -> None:
    """Move the accepted nodes' rows, slots start[b] + path[b][j] for j < n_accept[b], to slots
    start[b] + 1 + j in every layer of the cache (path [B, N], n_accept [B], start [B])."""
    B, N = path.shape
    cache._fits(B)
    _call("fe_cache_keep", t, _side(stream), lambda: (path, n_accept, start, *cache.tensors()), B, N, cache.n_layers,
          _ints(path, (B, N)), _ints(n_accept, (B,)), _ints(start, (B,)), ctypes.addressof(cache.kv), *cache.pages)
