"""Thin ctypes binding of the supervised head (``include/lc_head.h``): argument marshalling only.

As in :mod:`.binding`, every function takes torch tensors that live on the GPU, checks shape, dtype and contiguity, and passes
raw device pointers and the current HIP stream to the C entry point of the same name.  Results go into tensors the caller
brings; scratch (``ws``) is any GPU tensor of at least the size the ``*_workspace_bytes`` function of the operator gives.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

import torch

from . import binding as _b
from .binding import LC_F32, LC_BF16

LC_ACT_SIGMOID, LC_ACT_SILU, LC_ACT_GELU = 0, 1, 2

HEAD_EXPORTS = ("glu_workspace_bytes", "glu_fwd", "glu_bwd", "xent_workspace_bytes", "xent_fwd", "xent_fwd_bwd",
                "grad_clip_workspace_bytes", "grad_norm", "grad_clip")

__all__ = ["LC_ACT_SIGMOID", "LC_ACT_SILU", "LC_ACT_GELU", *HEAD_EXPORTS]

_typed = False


def _lib() -> C.CDLL:
    global _typed
    L = _b.lib()
    if not _typed:
        vp, i32, i64, f32, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
        L.glu_workspace_bytes.argtypes = [i32, i32, i32, C.c_int, C.c_int]
        L.glu_fwd.argtypes = [vp] * 5 + [i32, i32, i32, C.c_int, C.c_int, vp, sz, vp]
        L.glu_bwd.argtypes = [vp] * 8 + [i32, i32, i32, C.c_int, C.c_int, vp, sz, vp]
        L.xent_workspace_bytes.argtypes = [i32, i32, i32, C.c_int, C.c_int]
        L.xent_fwd.argtypes = [vp] * 6 + [i32, i32, i32, C.c_int, vp, sz, vp]
        L.xent_fwd_bwd.argtypes = [vp] * 8 + [i32, i32, i32, C.c_int, vp, sz, vp]
        L.grad_clip_workspace_bytes.argtypes = [i64, i32]
        L.grad_norm.argtypes = [vp, i32, vp, vp, sz, vp]
        L.grad_clip.argtypes = [vp, i32, f32, vp, vp, sz, vp]
        for name in HEAD_EXPORTS:
            getattr(L, name).restype = sz if name.endswith("_bytes") else C.c_int
        _typed = True
    return L


def _dev(t: Optional[torch.Tensor], shape, dtype, name: str) -> Optional[int]:
    """``binding._dev``; a tensor without values has no pointer."""
    return _b._dev(t, shape, dtype, name) or None


def glu_workspace_bytes(N: int, D: int, F: int, dtype: int = LC_F32, backward: bool = False) -> int:
    return int(_lib().glu_workspace_bytes(N, D, F, dtype, int(backward)))


def glu_fwd(x, wg, wu, h, gu, act: int, dtype: int = LC_F32, ws=None) -> None:
    (N, D), F = x.shape, wg.shape[0]
    dt = _b._op_dtype(dtype)
    wp, wb = _b._ws(ws)
    _b._check("glu_fwd", _lib().glu_fwd(
        _dev(x, (N, D), dt, "x"), _dev(wg, (F, D), dt, "wg"), _dev(wu, (F, D), dt, "wu"), _dev(h, (N, F), dt, "h"),
        _dev(gu, (N, 2, F), dt, "gu"), N, D, F, act, dtype, wp, wb, _b._stream()))


def glu_bwd(x, wg, wu, gu, dh, dx, dwg, dwu, act: int, dtype: int = LC_F32, ws=None) -> None:
    (N, D), F = x.shape, wg.shape[0]
    dt = _b._op_dtype(dtype)
    wp, wb = _b._ws(ws)
    _b._check("glu_bwd", _lib().glu_bwd(
        _dev(x, (N, D), dt, "x"), _dev(wg, (F, D), dt, "wg"), _dev(wu, (F, D), dt, "wu"),
        _dev(gu, (N, 2, F), dt, "gu"), _dev(dh, (N, F), dt, "dh"), _dev(dx, (N, D), dt, "dx"),
        _dev(dwg, (F, D), dt, "dwg"), _dev(dwu, (F, D), dt, "dwu"), N, D, F, act, dtype, wp, wb, _b._stream()))


def xent_workspace_bytes(N: int, D: int, V: int, dtype: int = LC_F32, grads: bool = False) -> int:
    return int(_lib().xent_workspace_bytes(N, D, V, dtype, int(grads)))


def xent_fwd(x, w, target, scale, loss, cost, dtype: int = LC_F32, ws=None) -> None:
    (N, D), V = x.shape, w.shape[0]
    dt = _b._op_dtype(dtype)
    wp, wb = _b._ws(ws)
    _b._check("xent_fwd", _lib().xent_fwd(
        _dev(x, (N, D), dt, "x"), _dev(w, (V, D), dt, "w"), _dev(target, (N,), torch.int64, "target"),
        _dev(scale, (N,), torch.float32, "scale"), _dev(loss, (N,), torch.float32, "loss"),
        _dev(cost, (1,), torch.float32, "cost"), N, D, V, dtype, wp, wb, _b._stream()))


def xent_fwd_bwd(x, w, target, scale, loss, cost, dx, dw, dtype: int = LC_F32, ws=None) -> None:
    (N, D), V = x.shape, w.shape[0]
    dt = _b._op_dtype(dtype)
    wp, wb = _b._ws(ws)
    _b._check("xent_fwd_bwd", _lib().xent_fwd_bwd(
        _dev(x, (N, D), dt, "x"), _dev(w, (V, D), dt, "w"), _dev(target, (N,), torch.int64, "target"),
        _dev(scale, (N,), torch.float32, "scale"), _dev(loss, (N,), torch.float32, "loss"),
        _dev(cost, (1,), torch.float32, "cost"), _dev(dx, (N, D), dt, "dx"), _dev(dw, (V, D), dt, "dw"), N, D, V, dtype,
        wp, wb, _b._stream()))


def grad_clip_workspace_bytes(tensors: Sequence[torch.Tensor]) -> int:
    return int(_lib().grad_clip_workspace_bytes(sum([t.numel() for t in tensors]), len(tensors)))


_VALUE_TYPES = {torch.float32: LC_F32, torch.bfloat16: LC_BF16}


def _tensor_list(src: Sequence[torch.Tensor], dst: Sequence[torch.Tensor]):
    """An array of lc_tensor_t: four 64-bit words each (src, dst, n, dtype in the low half of the last)."""
    if len(src) != len(dst):
        raise ValueError(f"{len(src)} tensors, but {len(dst)} to write to")
    words = []
    for a, b in zip(src, dst):
        kind = _VALUE_TYPES.get(a.dtype)
        if kind is None or b.dtype is not a.dtype:
            raise ValueError(f"tensors must be float32 or bfloat16 on both sides, got {a.dtype} and {b.dtype}")
        if not (a.is_cuda and b.is_cuda):
            raise ValueError("tensors must be GPU tensors")
        n = a.numel()
        if n != b.numel() or not (a.is_contiguous() and b.is_contiguous()):
            raise ValueError("tensors must be contiguous and of the same size on both sides")
        words += (a.data_ptr(), b.data_ptr(), n, kind)
    return (C.c_uint64 * len(words))(*words) if words else None


def grad_norm(tensors: Sequence[torch.Tensor], norm, ws=None) -> None:
    wp, wb = _b._ws(ws)
    _b._check("grad_norm", _lib().grad_norm(_tensor_list(tensors, tensors), len(tensors),
                                            _dev(norm, (1,), torch.float32, "norm"), wp, wb, _b._stream()))


def grad_clip(tensors: Sequence[torch.Tensor], out: Optional[Sequence[torch.Tensor]], max_norm: float, norm,
              ws=None) -> None:
    """``out`` None: in place."""
    wp, wb = _b._ws(ws)
    _b._check("grad_clip", _lib().grad_clip(_tensor_list(tensors, tensors if out is None else out), len(tensors), max_norm,
                                            _dev(norm, (1,), torch.float32, "norm"), wp, wb, _b._stream()))
