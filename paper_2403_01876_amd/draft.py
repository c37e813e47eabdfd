"""Python binding of the operators over drafted tokens of ``libdv.so``
(``include/dv_draft.h``): argument marshalling only, as in :mod:`.attn`.

``dv_attend_tree`` runs one layer's attention of drafted tokens that branch,
``dv_verify`` accepts drafts by the target model's logits and given random numbers,
``dv_keep_path`` moves the accepted ones together in the cache, and ``dv_quant_out``
reads cached tokens back as a 16-bit stream.  Tensors have to be on one GPU, or in pinned
memory of the host: others are refused.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import numpy as np
import torch

from .attn import (DV_BF16, DV_F16, QuantCache, _attend_args, _f32, _i32_t, _i64, _Q, _A, _u64,
                   _U, _vp)
from .dv import _addr, _check, _i32, _stream, lib

DV_F32 = 2
DV_MAX_DRAFTS = 128
_TYPES = {torch.float16: DV_F16, torch.bfloat16: DV_BF16, torch.float32: DV_F32}


class dv_verify_args(ctypes.Structure):
    _fields_ = [("type", _i32_t), ("batch", _i32_t), ("vocab", _i32_t), ("rows", _i32_t),
                ("logits", _vp), ("logits_row", _i64), ("drawn", _vp), ("drawn_row", _i64),
                ("parent", _vp), ("token", _vp), ("uniform", _vp), ("path", _vp), ("count", _vp),
                ("next", _vp), ("workspace", _vp), ("workspace_bytes", _u64)]


# Symbols include/dv_draft.h declares.
EXPORTS = ("dv_attend_tree", "dv_verify_bytes", "dv_verify", "dv_keep_path", "dv_quant_out")

_V = ctypes.POINTER(dv_verify_args)
for _name, _args in {
        "dv_attend_tree": [_Q, _i32_t, _i32_t, _vp, _vp, _vp, _A, _vp],
        "dv_verify_bytes": [_vp, _V, _U],
        "dv_verify": [_vp, _vp, _V, _vp],
        "dv_keep_path": [_Q, _i32_t, _i32_t, _i32_t, _vp, _vp, _vp, _vp, _vp],
        "dv_quant_out": [_Q, _i32_t, _i32_t, _i32_t, _vp, _vp, _vp, _u64, _i32_t, _U, _vp],
}.items():
    if not hasattr(lib, _name):
        raise ImportError(f"libdv.so lacks {_name}: rebuild with __graft_entry__.build()")
    _f = getattr(lib, _name)
    _f.argtypes = _args
    _f.restype = ctypes.c_int


def _array(name: str, x, dtype, least: int = 0):
    """The address of a contiguous device tensor of at least so many numbers."""
    if x.dtype is not dtype or not x.is_contiguous() or x.numel() < least:
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {least} numbers or more, "
                         f"got {tuple(x.shape)} {x.dtype}")
    return x.data_ptr()


def _astray(**tensors) -> str:
    """For a refusal's name, which tensors a GPU would not reach: those in the host's pageable
    memory, or on another GPU than the first that is on one.  Empty if there are none."""
    device, names = -1, []
    for name, x in tensors.items():
        if x is None or x.numel() == 0:
            continue
        at = x.get_device()
        if at < 0 and not x.is_pinned() or at >= 0 and device not in (-1, at):
            names.append(name)
        elif device < 0:
            device = at
    return f" ({', '.join(names)}: not in the GPU's memory)" if names else ""


def _lengths(name: str, x):
    """One-dimensional int32 lengths: the array, its address and size."""
    n = len(x)
    a, p = _i32(x, n)
    if a.ndim != 1 or a.size != n:
        raise ValueError(f"{name} must be one-dimensional, got {a.shape}")
    return a, p, n


def _temperatures(t, batch: int):
    """float32, one for each sequence."""
    if type(t) is not np.ndarray or t.dtype != np.float32 or t.shape != (batch,) or \
            not t.flags.c_contiguous:
        t = np.ascontiguousarray(np.broadcast_to(np.asarray(t, dtype=np.float32), (batch,)))
    return t


def dv_attend_tree(c: QuantCache, mb: int, layer: int, q_len, kv_len, parent, q, out,
                   scale: float, slopes=None, lse=None, workspace=None, stream=None,
                   check: bool = True) -> int:
    """As attn.dv_attend, of drafts that follow each other as ``parent`` (an int32 tensor
    [tokens]) says; ``workspace``: of attn.dv_attend_bytes bytes."""
    cache = c.cache.c
    a0, p0 = _i32(q_len, cache.batch)
    a1, p1 = _i32(kv_len, cache.batch)
    a = _attend_args(c, q, out, scale, slopes, None, lse, workspace)
    at = _array("parent", parent, torch.int32)
    a.rows = min(a.rows, parent.numel())
    name, d = "dv_attend_tree", q.get_device()
    # (the usual case asked for at once: a call is bound by the host where texts are short)
    if d < 0 or out.get_device() != d or parent.get_device() != d or \
            (slopes is not None and slopes.get_device() != d) or \
            (lse is not None and lse.get_device() != d) or \
            (workspace is not None and workspace.get_device() != d):
        name += _astray(q=q, out=out, parent=parent, slopes=slopes, lse=lse, workspace=workspace)
        if name != "dv_attend_tree":  # refused, after what else there is to refuse
            at = None
    rc = lib.dv_attend_tree(c.ref, mb, layer, p0, p1, at, ctypes.byref(a), _stream(stream))
    return _check(rc, name, check)


def _table(name: str, x, types):
    if x.dim() != 2 or x.dtype not in types or (x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError(f"{name} must be a tensor [drafts, vocab] of {tuple(types)} with contiguous "
                         f"rows, got {tuple(x.shape)} {x.dtype}")
    # (one row may have any stride)
    return x.data_ptr(), max(x.stride(0), x.shape[1]) if x.shape[0] < 2 else x.stride(0)


def dv_verify_bytes(q_len, logits, drawn: bool = False, check: bool = True):
    """Workspace bytes of a dv_verify with these lengths and logits' shape; ``drawn``:
    whether it will be given the drafts' distributions."""
    n, p, batch = _lengths("q_len", q_len)
    _table("logits", logits, _TYPES)
    a = dv_verify_args(type=_TYPES[logits.dtype], batch=batch, vocab=logits.shape[1],
                       drawn=16 if drawn else None)
    out = _u64(0)
    rc = lib.dv_verify_bytes(p, ctypes.byref(a), ctypes.byref(out))
    _check(rc, "dv_verify_bytes", check)
    return out.value if check else (rc, out.value)


def dv_verify(q_len, parent, token, logits, uniform, path, count, next, temperature=None,
              drawn=None, workspace=None, stream=None, check: bool = True) -> int:
    """Accept drafts of every sequence by the target's ``logits`` [drafts, vocab] (float16,
    bfloat16 or float32): ``parent``, ``token`` (int32) and ``uniform`` (float32) hold a number
    for each draft, ``drawn`` (float32 [drafts, vocab], or None) the distributions that those
    which follow them were drawn from, independently of each other.  ``path`` (int32 [drafts]), ``count`` and ``next`` (int32
    [batch]) receive the result.  ``temperature``: a number for all, or one for each sequence
    (host); ``workspace``: a tensor of dv_verify_bytes bytes."""
    n, p, batch = _lengths("q_len", q_len)
    la, lr = _table("logits", logits, _TYPES)
    rows, vocab = logits.shape
    da = dr = 0
    if drawn is not None:
        da, dr = _table("drawn", drawn, (torch.float32,))
        if drawn.shape[1] != vocab:
            raise ValueError(f"logits {tuple(logits.shape)}, drawn {tuple(drawn.shape)}")
        rows = min(rows, drawn.shape[0])
    rows = min(rows, parent.numel(), token.numel(), uniform.numel(), path.numel())
    ta = None
    if temperature is not None:
        t = _temperatures(temperature, batch)
        ta = t.ctypes.data
    wb = 0
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError(f"workspace must be contiguous, got strides {workspace.stride()}")
        wb = workspace.numel() * workspace.element_size()
    i32 = torch.int32
    a = dv_verify_args(_TYPES[logits.dtype], batch, vocab, rows, la, lr, da, dr,
                       _array("parent", parent, i32), _array("token", token, i32),
                       _array("uniform", uniform, torch.float32), _array("path", path, i32),
                       _array("count", count, i32, batch), _array("next", next, i32, batch),
                       _addr(workspace), wb)
    astray = _astray(logits=logits, drawn=drawn, parent=parent, token=token,
                     uniform=uniform, path=path, count=count, next=next, workspace=workspace)
    if astray:
        a.count = None
    rc = lib.dv_verify(p, ta, ctypes.byref(a), _stream(stream))
    return _check(rc, "dv_verify" + astray, check)


def dv_keep_path(c: QuantCache, mb: int, l0: int, l1: int, q_len, kv_len, path, count,
                 stream=None, check: bool = True) -> int:
    """Move the drafts that ``path`` and ``count`` (int32 tensors, as from dv_verify) name to
    the slots behind the tokens before the drafts."""
    batch = c.cache.c.batch
    a0, p0 = _i32(q_len, batch)
    a1, p1 = _i32(kv_len, batch)
    at = _array("path", path, torch.int32, 0 if a0 is None else sum(a0.tolist()))
    n = _array("count", count, torch.int32, batch)
    name = "dv_keep_path"
    if path.get_device() < 0 or path.get_device() != count.get_device():
        name += _astray(path=path, count=count)
        if name != "dv_keep_path":
            at = None
    rc = lib.dv_keep_path(c.ref, mb, l0, l1, p0, p1, at, n, _stream(stream))
    return _check(rc, name, check)


def dv_quant_out(src: QuantCache, mb: int, l0: int, l1: int, t0, t1, dst, dst_cap: int,
                 type: int, stream=None, check: bool = True):
    """Read tokens [t0, t1) back as a wire of 16-bit numbers (DV_F16 or DV_BF16); returns its
    bytes (with check=False: status and bytes)."""
    a0, p0 = _i32(t0, src.cache.c.batch)
    a1, p1 = _i32(t1, src.cache.c.batch)
    out, at, name = _u64(0), _addr(dst), "dv_quant_out"
    if isinstance(dst, np.ndarray) or isinstance(dst, torch.Tensor) and dst.get_device() < 0:
        name += _astray(dst=torch.as_tensor(dst))
        if name != "dv_quant_out":
            at = None
    rc = lib.dv_quant_out(src.ref, mb, l0, l1, p0, p1, at, dst_cap, type, ctypes.byref(out),
                          _stream(stream))
    _check(rc, name, check)
    return out.value if check else (rc, out.value)
