"""Weights in 4 bits over torch tensors: rounding by blocks of 32 columns, the way
back, and products of a few rows with such weights (declared in include/ws_fp4.h;
computed by the HIP kernels of libwsgemm.so, with no other path).

A linear layer y = x w^T, and a layer of experts, when tokens are decoded::

    W = quantize_weight(w)                        # w: out x in, or experts x out x in
    y = product(x, W)                             # x: tokens x in, bf16 or f16
    h = grouped_product(x, W, routes.offsets, index=routes.token)

Streams and errors as in ``fp8``; nothing here is recorded by autograd.  For many
rows (prompts, training) weights in 8 bits (``fp8``) are the faster ones.
"""
from __future__ import annotations

import ctypes

import torch

from . import wsgemm as _w
from .fp8 import E8M0, _Call, _check, _elsewhere, _index, _matrix, _mp, _need, _result, _raw_stream, _up

BLOCK = 32
_ROWS, _COLS = 16, 128  # of a tile


class ws_fp4_matrix(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("ld", ctypes.c_int64), ("ld_scales", ctypes.c_int64), ("batch", ctypes.c_int32),
                ("stride_codes", ctypes.c_int64), ("stride_scales", ctypes.c_int64)]


_lib = _w.library()
_p, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
_fp = ctypes.POINTER(ws_fp4_matrix)
for _name, _args, _res in (("ws_fp4_quantize", [_mp, _fp, _p], _i32), ("ws_fp4_dequantize", [_fp, _mp, _p], _i32),
                           ("ws_fp4_scales", [_fp, _p, _i64, _i64, _p], _i32),
                           ("ws_fp4_product_workspace", [_i64, _i64, _i64, _i32], _i64),
                           ("ws_fp4_product", [_mp, _p, _fp, _mp, _p, _i64, _p], _i32),
                           ("ws_fp4_grouped_product", [_mp, _p, _fp, _i32, _p, _mp, _p, _i64, _p], _i32)):
    getattr(_lib, _name).argtypes, getattr(_lib, _name).restype = _args, _res


class Fp4Matrix:
    """rows x cols in 4 bits, or a batch of such matrices (weights of experts).

    ``codes`` ((batch x) ceil(rows / 16) x pitch, uint8): tiles of 16 rows by 128
    columns, 1024 bytes each, in the order of include/ws_fp4.h.  ``packed_scales``
    ((batch x) ceil(rows / 16) x pitch, e8m0): their scales, 64 bytes for a tile;
    ``scales`` gives them by row.  Rows and columns are padded with zero codes and
    scales of 1; tiles of the next 16 rows may be further apart."""

    __slots__ = ("codes", "packed_scales", "rows", "cols", "_desc")

    def __init__(self, codes, scales, rows: int, cols: int):
        _need(codes, "codes", (torch.uint8,), (2, 3))
        _need(scales, "scales", (E8M0,), (codes.dim(),), codes.device)
        if rows < 0 or cols < 0:
            raise ValueError("%d x %d" % (rows, cols))
        cs, ss, shape, down, across = codes.stride(), scales.stride(), codes.shape, -(-rows // _ROWS), -(-cols // _COLS)
        batch = shape[0] if len(shape) == 3 else 1
        if shape[-2] != down or shape[-1] < 1024 * across or (shape[-1] > 1 and cs[-1] != 1):
            raise ValueError("codes %s of strides %s do not hold %d x %d values in tiles of 16 x 128" % (tuple(shape), cs, rows, cols))
        if tuple(scales.shape[:-1]) != tuple(shape[:-1]) or scales.shape[-1] < 64 * across or (scales.shape[-1] > 1 and ss[-1] != 1):
            raise ValueError("scales %s of strides %s: expected %s" % (tuple(scales.shape), ss, tuple(shape[:-1]) + (64 * across,)))
        ld = cs[-2] if down > 1 and shape[-1] > 0 else _up(shape[-1], 16)
        ld_scales = ss[-2] if down > 1 and scales.shape[-1] > 0 else _up(scales.shape[-1], 4)
        if ld % 16 or codes.data_ptr() % 16 or (batch > 1 and cs[0] % 16):
            raise ValueError("codes: tiles have to start at multiples of 16 bytes, got strides %s" % (cs,))
        if ld_scales % 4 or scales.data_ptr() % 4 or (batch > 1 and ss[0] % 4):
            raise ValueError("scales: tiles have to start at multiples of 4 bytes, got strides %s" % (ss,))
        if rows > 0 and cols > 0 and (ld < 1024 * across or ld_scales < 64 * across or (batch > 1 and (
                cs[0] < (down - 1) * ld + 1024 * across or ss[0] < (down - 1) * ld_scales + 64 * across))):
            raise ValueError("tiles and matrices may not overlap, got strides %s of codes and %s of scales" % (cs, ss))
        self.codes, self.packed_scales, self.rows, self.cols = codes, scales, rows, cols
        self._desc = ws_fp4_matrix(codes.data_ptr(), scales.data_ptr(), rows, cols, ld, ld_scales, batch,
                                   cs[0] if len(shape) == 3 else 0, ss[0] if len(shape) == 3 else 0)

    @property
    def batch(self):
        """Matrices of a batch, None for a single matrix."""
        return self.codes.shape[0] if self.codes.dim() == 3 else None

    @property
    def scales(self):
        """(batch x) rows x ceil(cols / 32), e8m0: the scale of every 32 columns of a row."""
        codes, cols = self.codes, -(-self.cols // BLOCK)
        if _elsewhere(codes, None):
            with _Call(codes.device, None, []):
                return self.scales
        out = torch.empty(codes.shape[:-2] + (self.rows, cols), dtype=E8M0, device=codes.device)
        _check(_lib.ws_fp4_scales(self._desc, out.data_ptr(), cols, self.rows * cols, _raw_stream(codes.device.index)), "ws_fp4_scales")
        return out

    @classmethod
    def empty(cls, rows: int, cols: int, batch: int | None = None, device="cuda"):
        if rows < 0 or cols < 0:
            raise ValueError("%d x %d" % (rows, cols))
        down, across, lead = -(-rows // _ROWS), -(-cols // _COLS), () if batch is None else (batch,)
        q = object.__new__(cls)
        q.codes = codes = torch.empty(lead + (down, 1024 * across), dtype=torch.uint8, device=device)
        q.packed_scales = scales = torch.empty(lead + (down, 64 * across), dtype=E8M0, device=device)
        q.rows, q.cols = rows, cols
        q._desc = ws_fp4_matrix(codes.data_ptr(), scales.data_ptr(), rows, cols, 1024 * across, 64 * across, 1 if batch is None else batch,
                                down * 1024 * across, down * 64 * across)
        return q

    def dequantize(self, out_dtype: str = "f32", out=None, stream=None):
        """The values, exactly ("f32", "bf16"; bf16 from 2^-126 up)."""
        shape = (() if self.batch is None else (self.batch,)) + (self.rows, self.cols)
        if out_dtype == "f16" or (out is not None and out.dtype == torch.float16):
            raise ValueError("binary16 does not hold the values")
        codes = self.codes
        if _elsewhere(codes, stream):
            with _Call(codes.device, stream, [codes, self.packed_scales, out]):
                return self.dequantize(out_dtype, out)
        out, m = _result(out, out_dtype, shape, codes.device)
        _check(_lib.ws_fp4_dequantize(self._desc, m, _raw_stream(codes.device.index)), "ws_fp4_dequantize")
        return out


def quantize_weight(w, out: Fp4Matrix | None = None, stream=None) -> Fp4Matrix:
    """w (out x in, or experts x out x in; f32, bf16 or f16) in 4 bits, with a scale for
    every 32 columns of a row."""
    m = _matrix(w, "w", (2, 3))
    if _elsewhere(w, stream):
        with _Call(w.device, stream, [w] + ([out.codes, out.packed_scales] if out is not None else [])):
            return quantize_weight(w, out)
    batch = m.batch if w.dim() == 3 else None
    if out is None:
        out = Fp4Matrix.empty(m.rows, m.cols, batch, w.device)
    elif (out.rows, out.cols, out.batch) != (m.rows, m.cols, batch) or out.codes.device != w.device:
        raise ValueError("out: expected %s x %d x %d on %s" % (batch, m.rows, m.cols, w.device))
    _check(_lib.ws_fp4_quantize(m, out._desc, _raw_stream(w.get_device())), "ws_fp4_quantize")
    return out


def _rows(A, B, index):
    """A's descriptor, the address of index and the rows of the result."""
    m = _matrix(A, "A", device=B.codes.device)
    if A.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("A: expected bf16 or f16, got %s" % A.dtype)
    if m.cols != B.cols:
        raise ValueError("A (%d x %d) and B (%d x %d) have to have as many columns" % (m.rows, m.cols, B.rows, B.cols))
    rows = m.rows if index is None else index.numel()
    return m, 0 if index is None else _index(index, "index", rows, A.device), rows


def _work(rows, B, groups, A):
    """Work memory of a product and its size."""
    if rows <= 16 * max(groups, 1):  # none: not asked for, as these are the shortest calls
        return None, 0
    need = _lib.ws_fp4_product_workspace(rows, B.rows, B.cols, groups)
    return (torch.empty(need, dtype=torch.uint8, device=A.device) if need > 0 else None), max(need, 0)


def product(A, B: Fp4Matrix, C=None, out_dtype: str = "bf16", index=None, stream=None):
    """A B^T: A is rows x K in bf16 or f16, B is N x K in 4 bits; sums in binary32,
    rounded once to C (its type counts) or a new tensor of out_dtype ("f32", "bf16",
    "f16").  index (int32): the source row of each result row; out of range, zeros."""
    if B.batch is not None:
        raise ValueError("B has to be a single matrix")
    m, at, rows = _rows(A, B, index)
    if _elsewhere(A, stream):
        with _Call(A.device, stream, [A, B.codes, B.packed_scales, C, index]):
            return product(A, B, C, out_dtype, index)
    C, mc = _result(C, out_dtype, (rows, B.rows), A.device)
    work, need = _work(rows, B, -1, A)
    _check(_lib.ws_fp4_product(m, at, B._desc, mc, work.data_ptr() if need else 0, need, _raw_stream(A.get_device())), "ws_fp4_product")
    return C


def grouped_product(A, B: Fp4Matrix, offsets, C=None, out_dtype: str = "bf16", index=None, stream=None):
    """Rows offsets[g] .. offsets[g + 1] - 1 (of A, or of index's rows of A) times
    B[g]^T; rows in no group, before the first or after the last, become zeros.
    offsets: int32 on the device, not decreasing.  Sums as in product."""
    if B.batch is None:
        raise ValueError("B has to be a batch")
    m, at, rows = _rows(A, B, index)
    if _elsewhere(A, stream):
        with _Call(A.device, stream, [A, B.codes, B.packed_scales, offsets, C, index]):
            return grouped_product(A, B, offsets, C, out_dtype, index)
    _need(offsets, "offsets", (torch.int32,), (1,), A.device)
    off = _index(offsets, "offsets", B.batch + 1, A.device)
    C, mc = _result(C, out_dtype, (rows, B.rows), A.device)
    work, need = _work(rows, B, B.batch, A)
    _check(_lib.ws_fp4_grouped_product(m, at, B._desc, B.batch, off, mc, work.data_ptr() if need else 0, need,
                                       _raw_stream(A.get_device())), "ws_fp4_grouped_product")
    return C
