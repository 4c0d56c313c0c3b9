"""Matrices in 8-bit floating point with a scale for each block of 128 channels: encoding and product
(``include/codecgauge_block8.h``).

Bindings of the C entry points with the same names, in the manner of ``paged.py``. A coded matrix is a pair of
tensors: codes float8_e4m3fn [R][K] and scales float32 [ceil(R / rows)][ceil(K / 128)], rows 1 or 128.
"""
from __future__ import annotations

import torch

from . import _check
from . import paged as _p

BLOCK = 128
_E4M3 = torch.float8_e4m3fn


def _matrix(name: str, t, R: int, K: int, dtype, dev: int):
    """Checks a matrix [R][K] on the device whose rows are contiguous; its address and row stride (0 for at most one row)."""
    if t.shape != (R, K):
        _p._bad(f"{name}: expected shape [{R}, {K}], got {list(t.shape)}")
    if t.dtype is not dtype or t.get_device() != dev:
        _p._bad(f"{name}: expected a {dtype} matrix on device {dev}")
    row, one = t.stride()
    if one != 1 and K > 1:
        _p._bad(f"{name}: the last dimension must be contiguous")
    return t.data_ptr(), (row if R > 1 else 0)


def _shape(name: str, t):
    if t.dim() != 2:
        _p._bad(f"{name}: expected a matrix, got {list(t.shape)}")
    return t.shape


def _scales(name: str, t, R: int, K: int, rows: int, dev: int) -> int:
    shape = (-(-R // rows), -(-K // BLOCK))
    if t.shape != shape or t.dtype is not torch.float32 or t.get_device() != dev or not t.is_contiguous():
        _p._bad(f"{name}: expected a contiguous float32 tensor {list(shape)} on device {dev}")
    return t.data_ptr()


def block8_encode(x, codes, scales, rows: int = 1, stream=None) -> None:
    """codes and scales of x [R][K] (bf16 or fp16, K a multiple of 16; rows may have a stride), a scale for each
    128 channels of a row (rows=1: activations) or of 128 rows (rows=128: weights) (cg_block8_encode)."""
    dev = _p._device()
    if dev >= 0 and _p._took("block8_encode", x, codes, scales, rows, dev, _p._stream(stream)):
        return
    if rows not in (1, BLOCK):
        _p._bad(f"rows={rows}: must be 1 or {BLOCK}")
    elem, (R, K) = _p._elem(x), _shape("x", x)
    xp, xs = _matrix("x", x, R, K, x.dtype, dev)
    cp, cs = _matrix("codes", codes, R, K, _E4M3, dev)
    _check(_p._fn("cg_block8_encode")(elem, R, K, rows, xp, xs, cp, cs, _scales("scales", scales, R, K, rows, dev), _p._stream(stream)))


def block8_matmul(x, x_scales, w, w_scales, out, stream=None) -> None:
    """out [M][N] (bf16 or fp16; rows may have a stride) = x w^T of the coded matrices x [M][K] (rows=1) and
    w [N][K] (rows=128) (cg_block8_matmul)."""
    dev = _p._device()
    if dev >= 0 and _p._took("block8_matmul", x, x_scales, w, w_scales, out, dev, _p._stream(stream)):
        return
    elem, (M, K), N = _p._elem(out), _shape("x", x), _shape("w", w)[0]
    xp, xs = _matrix("x", x, M, K, _E4M3, dev)
    wp, ws = _matrix("w", w, N, K, _E4M3, dev)
    op, os = _matrix("out", out, M, N, out.dtype, dev)
    _check(_p._fn("cg_block8_matmul")(elem, M, N, K, xp, xs, _scales("x_scales", x_scales, M, K, 1, dev), wp, ws,
                                      _scales("w_scales", w_scales, N, K, BLOCK, dev), op, os, _p._stream(stream)))
