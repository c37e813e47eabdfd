"""Python binding of the 8-bit cache operators of ``libdv.so``
(``include/dv_attn.h``): argument marshalling only, as in :mod:`.dv`.

A :class:`QuantCache` is a :class:`dv.Cache` with ``elem_bytes=1`` plus its scale
arrays (and, optionally, weights and positions).  ``dv_quant_in`` appends a
16-bit stream to it, ``dv_attend`` runs one layer's attention over it and
``dv_evict`` compacts it by accumulated weight.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from .dv import (Cache, _addr, _check, _i32, _stream, dv_cache, lib)

DV_F16, DV_BF16 = 0, 1
_TYPES = {torch.float16: DV_F16, torch.bfloat16: DV_BF16}

_pp = ctypes.POINTER(ctypes.c_void_p)
_i32_t, _i64, _f32, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p
_u64 = ctypes.c_uint64


class dv_quant(ctypes.Structure):
    _fields_ = [("cache", ctypes.POINTER(dv_cache)), ("scale_block", _i32_t), ("scale", _pp),
                ("weight", _pp), ("position", _pp)]


class dv_attend_args(ctypes.Structure):
    _fields_ = [("type", _i32_t), ("q_heads", _i32_t), ("scale", _f32), ("decay", _f32),
                ("weigh", _i32_t), ("rows", _i32_t), ("q", _vp), ("out", _vp),
                ("q_token", _i64), ("q_head", _i64), ("out_token", _i64), ("out_head", _i64),
                ("slopes", _vp), ("lse", _vp), ("workspace", _vp), ("workspace_bytes", _u64)]


# Symbols include/dv_attn.h declares.
EXPORTS = ("dv_quant_scale_bytes", "dv_quant_in", "dv_attend_bytes", "dv_attend", "dv_evict")

_Q, _A, _U = ctypes.POINTER(dv_quant), ctypes.POINTER(dv_attend_args), ctypes.POINTER(_u64)
for _name, _args in {
        "dv_quant_scale_bytes": [_Q, _U],
        "dv_quant_in": [_Q, _i32_t, _i32_t, _i32_t, _vp, _vp, _vp, _u64, _i32_t, _vp],
        "dv_attend_bytes": [_Q, _vp, _vp, _A, _U],
        "dv_attend": [_Q, _i32_t, _i32_t, _vp, _vp, _A, _vp],
        "dv_evict": [_Q, _i32_t, _Q, _i32_t, _i32_t, _i32_t, _vp, _vp, _i32_t, _vp, _i32_t, _vp],
}.items():
    if not hasattr(lib, _name):
        raise ImportError(f"libdv.so lacks {_name}: rebuild with __graft_entry__.build()")
    _f = getattr(lib, _name)
    _f.argtypes = _args
    _f.restype = ctypes.c_int


_attend, _byref = lib.dv_attend, ctypes.byref


class QuantCache:
    """A ``dv_quant`` descriptor plus what it points to.

    ``cache``: a dense or paged ``dv.Cache`` with ``elem_bytes=1``.  ``scales``,
    ``weights`` and ``positions``: one device array for each microbatch (entries of
    the last two may be None); ``scale_block``: tokens that share a scale (the
    block size of a paged cache, which is the default there)."""

    def __init__(self, cache: Cache, scales: Sequence, scale_block: int = 0,
                 weights: Optional[Sequence] = None, positions: Optional[Sequence] = None):
        self.cache = cache
        self.scale_block = scale_block or cache.c.block_size
        self._keep = []
        arrays = []
        for name, arr in (("scales", scales), ("weights", weights), ("positions", positions)):
            if arr is None:
                arrays.append(None)
                continue
            if len(arr) != len(cache.bases):
                raise ValueError(f"{name} has {len(arr)} entries, the cache has "
                                 f"{len(cache.bases)} microbatches")
            self._keep += [x for x in arr if x is not None and not isinstance(x, int)]
            arrays.append((_vp * len(arr))(*[_addr(x) for x in arr]))
        self._arrays = arrays
        self.c = dv_quant(ctypes.pointer(cache.c), self.scale_block,
                          *[None if a is None else ctypes.cast(a, _pp) for a in arrays])
        self.ref = ctypes.byref(self.c)


def dv_quant_scale_bytes(c: QuantCache, check: bool = True):
    out = _u64(0)
    rc = lib.dv_quant_scale_bytes(c.ref, ctypes.byref(out))
    _check(rc, "dv_quant_scale_bytes", check)
    return out.value if check else (rc, out.value)


def dv_quant_in(dst: QuantCache, mb: int, l0: int, l1: int, t0, t1, src, src_bytes: int,
                type: int, stream=None, check: bool = True) -> int:
    """Append tokens [t0, t1) from a wire of 16-bit numbers (DV_F16 or DV_BF16)."""
    a0, p0 = _i32(t0, dst.cache.c.batch)
    a1, p1 = _i32(t1, dst.cache.c.batch)
    rc = lib.dv_quant_in(dst.ref, mb, l0, l1, p0, p1, _addr(src), src_bytes, type,
                         _stream(stream))
    return _check(rc, "dv_quant_in", check)


def _rows(name: str, x, dim: int):
    """A [tokens, heads, head_dim] tensor's tokens, heads and strides."""
    shape, strides = x.shape, x.stride()
    if len(shape) != 3 or shape[2] != dim or strides[2] != 1 or x.dtype not in _TYPES:
        raise ValueError(f"{name} must be a float16 or bfloat16 tensor [tokens, heads, {dim}] "
                         f"with contiguous rows, got {tuple(shape)} {x.dtype}")
    return shape[0], shape[1], strides[0], strides[1]


def _floats(name: str, x, shape):
    if x.dtype is not torch.float32 or x.dim() != len(shape) or x.shape[-1] != shape[-1] or \
            not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 tensor of {shape}, got "
                         f"{tuple(x.shape)} {x.dtype}")


def dv_attend_bytes(c: QuantCache, q_len, kv_len, q, weights: bool = False,
                    check: bool = True):
    """Workspace bytes of a dv_attend of these lengths and queries' shape;
    ``weights``: whether it will accumulate them."""
    batch = c.cache.c.batch
    a0, p0 = _i32(q_len, batch)
    a1, p1 = _i32(kv_len, batch)
    _rows("q", q, c.cache.c.head_dim)
    a = dv_attend_args(type=_TYPES[q.dtype], q_heads=q.shape[1], weigh=int(weights))
    out = _u64(0)
    rc = lib.dv_attend_bytes(c.ref, p0, p1, ctypes.byref(a), ctypes.byref(out))
    _check(rc, "dv_attend_bytes", check)
    return out.value if check else (rc, out.value)


def _attend_args(c: QuantCache, q, out, scale, slopes, decay, lse, workspace):
    dim = c.cache.c.head_dim
    rows, heads, qt, qh = _rows("q", q, dim)
    out_rows, out_heads, ot, oh = _rows("out", out, dim)
    if out_heads != heads or out.dtype is not q.dtype:
        raise ValueError(f"q {tuple(q.shape)} {q.dtype}, out {tuple(out.shape)} {out.dtype}")
    if out_rows < rows:
        rows = out_rows
    if slopes is not None:
        _floats("slopes", slopes, (heads,))
        slopes = slopes.data_ptr()
    if lse is not None:
        _floats("lse", lse, (min(rows, lse.shape[0]), heads))
        rows, lse = min(rows, lse.shape[0]), lse.data_ptr()
    wb = 0
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError(f"workspace must be contiguous, got strides {workspace.stride()}")
        wb = workspace.numel() * workspace.element_size()
    return dv_attend_args(_TYPES[q.dtype], heads, scale, 0.0 if decay is None else decay,
                          decay is not None, rows, q.data_ptr(), out.data_ptr(), qt, qh, ot, oh,
                          slopes, lse, _addr(workspace), wb)


def dv_attend(c: QuantCache, mb: int, layer: int, q_len, kv_len, q, out, scale: float,
              slopes=None, decay: Optional[float] = None, lse=None, workspace=None, stream=None,
              check: bool = True) -> int:
    """Attention of the queries ``q`` [tokens, q_heads, head_dim] into ``out`` (any
    strides that are multiples of 8, rows contiguous).  ``decay``: accumulate
    the cache's weights, those from before times this (None: do not).  ``lse``: a
    float32 [tokens, q_heads] tensor.  ``workspace``: a tensor of dv_attend_bytes
    bytes."""
    cache = c.cache.c
    a0, p0 = _i32(q_len, cache.batch)
    a1, p1 = _i32(kv_len, cache.batch)
    a = _attend_args(c, q, out, scale, slopes, decay, lse, workspace)
    rc = _attend(c.ref, mb, layer, p0, p1, _byref(a), _stream(stream))
    return _check(rc, "dv_attend", check)


def dv_evict(src: QuantCache, src_mb: int, dst: QuantCache, dst_mb: int, l0: int, l1: int,
             length, keep, recent: int, kept, kept_stride: Optional[int] = None, stream=None,
             check: bool = True) -> int:
    """Keep min(length, keep) tokens of each head; ``kept``: an int32 device tensor
    [l1 - l0, batch, heads, kept_stride] that receives their slots."""
    batch = src.cache.c.batch
    a0, p0 = _i32(length, batch)
    a1, p1 = _i32(keep, batch)
    if kept_stride is None:
        want = (l1 - l0, batch, src.cache.c.num_heads)
        if kept.dtype != torch.int32 or not kept.is_contiguous() or kept.shape[:-1] != want:
            raise ValueError(f"kept must be a contiguous int32 tensor {want} + (slots,), got "
                             f"{tuple(kept.shape)} {kept.dtype}")
        kept_stride = kept.shape[-1]
    rc = lib.dv_evict(src.ref, src_mb, dst.ref, dst_mb, l0, l1, p0, p1, recent, _addr(kept),
                      kept_stride, _stream(stream))
    return _check(rc, "dv_evict", check)
