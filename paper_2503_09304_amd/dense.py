"""The dense calls of libqmoe.so (include/qdense.h) on torch tensors: argument marshalling only.

Rows are tensors [tokens, dim], or [tokens, heads, dim] where heads are normalised by themselves, with any strides of tokens and heads
that are multiples of 16 bytes (dense_linear's output: any) and dense elements.  Outputs are the caller's tensors.  All tensors of a call are on one
device, which need not be the current one; the call enqueues on PyTorch's current stream of that device.  A tensor that belongs to
another stream's work is the caller's to order, as with any kernel."""
from __future__ import annotations

import ctypes as C
import struct
import threading
from typing import Optional

import torch

from .attention import _bad, _device, _enqueue, _long, _whole
from .binding import MOE_E_ARG, MoeError, lib

DENSE_BF16, DENSE_F32, DENSE_FP8 = 0, 1, 2
_TYPES = {torch.bfloat16: DENSE_BF16, torch.float32: DENSE_F32, torch.float8_e4m3fn: DENSE_FP8, torch.uint8: DENSE_FP8}


class _Matrix(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("rows", C.c_int32), ("cols", C.c_int32)]


# dense_rows are passed as slices of one array of 64-bit numbers, a thread's own, written anew by every call (data, scale, two strides, type).
_ROWS = 5
_pack = [None] + [struct.Struct(f"{_ROWS * n}q").pack_into for n in (1, 2, 3, 4)]


class _Numbers(threading.local):
    def __init__(self):
        self.to = (C.c_int64 * (4 * _ROWS))()
        self.at = C.addressof(self.to)


_numbers = _Numbers()
_ready = None


def _lib():
    global _ready
    if _ready is None:
        L = lib()
        P, I, F, Z = C.c_void_p, C.c_int32, C.c_float, C.c_size_t
        L.dense_norm.argtypes = [P, P, P, P, P, I, F, F, I, I, I, P]
        L.dense_pack4.argtypes = [P, P, P, P]
        L.dense_linear.argtypes = [P, P, P, I, P, Z, P]
        for f in ("dense_norm", "dense_pack4", "dense_linear"):
            getattr(L, f).restype = I
        for f, n in (("dense_matrix4_code_bytes", 2), ("dense_matrix4_scale_bytes", 2), ("dense_linear_workspace_bytes", 5)):
            getattr(L, f).argtypes = [I] * n
            getattr(L, f).restype = Z
        _ready = L
    return _ready


def _rows(t, name: str, shape, dev: int, types, scale=None):
    """A tensor of this shape on this device as dense_rows; shape [T, D] or [T, H, D]."""
    if t.dtype not in types or t.shape != shape or t.get_device() != dev:
        _bad(f"{name} must be a tensor {list(shape)} of {' or '.join(str(d) for d in types)} on GPU {dev}, not {t.dtype} {list(t.shape)} on {t.device}")
    s = t.stride()
    if s[-1] != 1 and shape[-1] > 1:
        _bad(f"the elements of a row of {name} must be dense")
    kind = _TYPES[t.dtype]
    at = 0
    if kind == DENSE_FP8:
        if scale is None:
            _bad(f"8-bit rows need a scale ({name})")
        at = _whole(scale, f"the scale of {name}", torch.uint8, (*shape[:-1], shape[-1] // 32), dev)
    elif scale is not None:
        _bad(f"{name} is not in 8 bits and has no scale")
    return t.data_ptr(), at, s[0] if shape[0] > 1 else 0, s[1] if len(shape) == 3 and shape[1] > 1 else 0, kind


_X, _ADD, _OUT = (torch.bfloat16,), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.float8_e4m3fn, torch.uint8)


def dense_norm(x, weight, out, eps: float = 1e-6, add=None, total=None, scale=None, shift: float = 0.0) -> int:
    """r = x + add, total = r, out = r / sqrt(mean(r^2) + eps) * (weight + shift), for rows [tokens, dim] or heads [tokens, heads, dim].  x bfloat16; add, total
    bfloat16 or float32 (total may be add), or None; weight [dim] bfloat16 or float32, or None; out bfloat16, or float8_e4m3fn (or its bytes as uint8) with
    scale uint8 [.., dim/32]."""
    shape = x.shape
    if len(shape) not in (2, 3):
        _bad("x must be [tokens, dim] or [tokens, heads, dim]")
    if max(shape) >> 31:
        _long("x")
    dev = _device(x, "x")
    L, w = _lib(), _numbers
    r = [*_rows(x, "x", shape, dev, _X), *_rows(out, "out", shape, dev, _OUT, scale)]
    at = w.at
    if add is not None:
        r += _rows(add, "add", shape, dev, _ADD)
        if total is not None:
            r += _rows(total, "total", shape, dev, (add.dtype,))
    elif total is not None:
        _bad("total needs add")
    _pack[len(r) // _ROWS](w.to, 0, *r)
    wt = DENSE_BF16
    if weight is not None:
        if weight.dtype not in _ADD:
            _bad("weight must be bfloat16 or float32")
        wt = _TYPES[weight.dtype]
        weight = _whole(weight, "weight", weight.dtype, shape[-1:], dev)
    return _enqueue(L.dense_norm, dev, at, at + 80 if add is not None else None, at + 120 if total is not None else None, at + 40, weight, wt, shift, eps,
                    shape[0], shape[1] if len(shape) == 3 else 1, shape[-1])


class DenseMatrix4:
    """A matrix [rows, cols] of 4-bit weights: codes uint8 [rows, cols/2] (e2m1, the even column in the low nibble), scales uint8 [rows, cols/32] (e8m0).  Packs
    them into memory of its own, on the current stream."""

    def __init__(self, codes, scales):
        if codes.dim() != 2 or codes.shape[0] >> 31 or codes.shape[1] >> 30:
            _bad("codes must be [rows, cols/2]")
        self.rows, self.cols = codes.shape[0], 2 * codes.shape[1]
        self._device = d = _device(codes, "codes")
        L = _lib()
        nc, ns = (int(f(self.rows, self.cols)) for f in (L.dense_matrix4_code_bytes, L.dense_matrix4_scale_bytes))
        if nc == 0:
            raise MoeError(MOE_E_ARG, L.moe_last_error().decode())
        src = _whole(codes, "codes", torch.uint8, (self.rows, self.cols // 2), d), _whole(scales, "scales", torch.uint8, (self.rows, self.cols // 32), d)
        self.codes, self.scales = (torch.empty(n, dtype=torch.uint8, device=codes.device) for n in (nc, ns))
        self._c = _Matrix(self.codes.data_ptr(), self.scales.data_ptr(), self.rows, self.cols)
        self._at = C.addressof(self._c)
        _enqueue(L.dense_pack4, d, *src, self._at)


_LIN_X, _LIN_OUT = (torch.bfloat16, torch.float8_e4m3fn, torch.uint8), (torch.bfloat16, torch.float32)


def dense_linear(x, matrix: DenseMatrix4, out, scale=None) -> int:
    """out [tokens, rows] = x [tokens, cols] times the matrix, transposed.  x bfloat16, or float8_e4m3fn (or its bytes as uint8) with scale uint8 [tokens, cols/32], as
    dense_norm writes them; out bfloat16 or float32.  Where the sums are cut into ranges of columns the call takes scratch memory from PyTorch's allocator,
    for the time of its kernels."""
    if x.dim() != 2:
        _bad("x must be [tokens, cols]")
    T, dev = x.shape[0], matrix._device
    if T >> 31:
        _long("x")
    L, w = _lib(), _numbers
    r = (*_rows(x, "x", (T, matrix.cols), dev, _LIN_X, scale), *_rows(out, "out", (T, matrix.rows), dev, _LIN_OUT))
    nb = L.dense_linear_workspace_bytes(T, matrix.rows, matrix.cols, r[4], r[9])
    ws = None if nb == 0 else torch.empty(nb, dtype=torch.uint8, device=x.device)
    _pack[2](w.to, 0, *r)
    return _enqueue(L.dense_linear, dev, w.at, matrix._at, w.at + 40, T, None if ws is None else ws.data_ptr(), nb)
