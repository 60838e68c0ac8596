"""The 8-bit path over torch tensors: quantisation by blocks, the block-scaled
product and its grouped forms (declared in include/ws_fp8.h; computed by the HIP
kernels of libwsgemm.so, with no other path).

A linear layer y = x w^T in 8 bits, forward and backward::

    xq, xq_t = quantize_both(x)               # x: tokens x in
    wq, wq_t = quantize_weight(w)             # w: out x in
    y = product(xq, wq)                       # tokens x out
    gq, gq_t = quantize_both(dy)
    dx = product(gq, wq_t)                    # tokens x in
    dw = product(gq_t, xq_t, out_dtype="f32") # out x in

Codes are torch.float8_e4m3fn, scales torch.float8_e8m0fnu (powers of two) for
128 columns of a row, or of 128 rows (weights).

Calls enqueue on ``stream`` (default: the current stream of the operands'
device) and return at once.  Results and work memory made here belong to that
stream; tensors handed in with a ``stream`` are marked as in use by it, so that
their memory is not given out again before the work is done (on the current
stream that is the caller's, as for torch's own operations).  Sizes, types, devices and
strides are checked and raise ValueError, a status of the library raises
WsGemmError; the contents of codes, scales and offsets are not looked at.
Nothing here is recorded by autograd: a layer's backward makes the gradients with
the calls above.
"""
from __future__ import annotations

import contextlib
import ctypes

import torch

from . import wsgemm as _w

BLOCK = 128
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
_MOST = 1 << 30  # rows or columns that the library takes; counts have to fit before ctypes cuts them
_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_CODES = {torch.float32: _w.WS_OUT_F32, torch.bfloat16: _w.WS_OUT_BF16, torch.float16: _w.WS_OUT_F16}


class ws_fp8_matrix(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("ld", ctypes.c_int64), ("ld_scales", ctypes.c_int64), ("block_rows", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("stride_codes", ctypes.c_int64), ("stride_scales", ctypes.c_int64)]


class ws_matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("ld", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("batch", ctypes.c_int32), ("stride", ctypes.c_int64)]


class ws_fp8_kernel_info(ctypes.Structure):
    _fields_ = [("tile_m", ctypes.c_int32), ("tile_n", ctypes.c_int32), ("stages", ctypes.c_int32), ("launch", ctypes.c_int32),
                ("rows", ctypes.c_int64)]


_lib = _w.library()
_p, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
_mp, _qp = ctypes.POINTER(ws_matrix), ctypes.POINTER(ws_fp8_matrix)
for _name, _args, _res in (
        ("ws_fp8_quantize_rows", [_mp, _p, _qp, _p], _i32),
        ("ws_fp8_quantize_both", [_mp, _p, _i32, _p, _qp, _qp, _p], _i32),
        ("ws_fp8_padded_blocks", [_i64, _i32], _i64),
        ("ws_fp8_quantize_weight", [_mp, _qp, _qp, _p], _i32),
        ("ws_fp8_plan", [_i64, _i64, _i64, _i32, _i32, _i32, ctypes.POINTER(ws_fp8_kernel_info), ctypes.POINTER(_i32)], _i32),
        ("ws_fp8_product", [_qp, _qp, _f32, _f32, _mp, _mp, _p], _i32),
        ("ws_fp8_grouped_product", [_qp, _qp, _i32, _p, _f32, _mp, _p], _i32),
        ("ws_fp8_grouped_gradient", [_qp, _qp, _i64, _i32, _p, _f32, _f32, _mp, _mp, _p], _i32)):
    getattr(_lib, _name).argtypes, getattr(_lib, _name).restype = _args, _res

_ws_fp8_product, _ws_fp8_quantize_rows = _lib.ws_fp8_product, _lib.ws_fp8_quantize_rows
_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice


def _up(n: int, m: int) -> int:
    return -(-n // m) * m


def _check(status: int, where: str) -> None:
    if status != _w.WS_OK:
        raise _w.WsGemmError(where, status)


class _Call:
    """Makes a call's stream and device the current ones, so that its results and
    work memory belong to it, and marks tensors of the device as in use by it (what
    else was handed in is refused by the call's own checks)."""

    __slots__ = ("_device", "_stream", "_tensors", "_stack")

    def __init__(self, device: torch.device, stream, tensors):
        if stream is not None and stream.device != device:
            raise ValueError("the stream belongs to %s, the tensors to %s" % (stream.device, device))
        self._device, self._stream, self._tensors = device, stream, tensors

    def __enter__(self):
        with contextlib.ExitStack() as stack:  # left again where something fails
            stack.enter_context(torch.cuda.device(self._device))
            if self._stream is not None:
                stack.enter_context(torch.cuda.stream(self._stream))
                for t in self._tensors:
                    if isinstance(t, torch.Tensor) and t.is_cuda and t.device == self._device:
                        t.record_stream(self._stream)
            self._stack = stack.pop_all()
        return self

    def __exit__(self, *exc):
        self._stack.close()


def _elsewhere(t, stream):
    """Whether a call on t does not use the current stream of t's device, or that is
    not the current device: then it is made again inside a _Call."""
    return stream is not None or t.get_device() != _current_device()


def _need(t, what: str, dtypes, dims, device=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("%s: expected a cuda tensor" % what)
    if t.dtype not in dtypes or t.dim() not in dims:
        raise ValueError("%s: expected %s of %s dimensions, got %s %s" % (what, "/".join(map(str, dtypes)),
                                                                         "/".join(map(str, dims)), t.dtype, tuple(t.shape)))
    if device is not None and t.device != device:
        raise ValueError("%s: on %s, the other operands on %s" % (what, t.device, device))


def _matrix(t, what: str, dims=(2,), device=None) -> ws_matrix:
    """Descriptor of a float tensor (batch x) rows x cols whose columns lie next to each other."""
    code = _CODES.get(t.dtype) if isinstance(t, torch.Tensor) else None
    if code is None or not t.is_cuda or t.dim() not in dims or (device is not None and t.device != device):
        _need(t, what, _CODES, dims, device)
    shape, stride = t.shape, t.stride()
    if len(shape) == 2:
        rows, cols = shape
        ld = stride[0]
        if rows <= 1:
            ld = cols
        if cols > 1 and stride[1] != 1 or ld < cols:
            raise ValueError("%s: columns have to lie next to each other and rows may not overlap, got strides %s" % (what, stride))
        return ws_matrix(t.data_ptr(), rows, cols, ld, code, 1, 0)
    batch, rows, cols = shape
    ld = stride[1] if rows > 1 else cols
    if cols > 1 and stride[2] != 1 or ld < cols or (batch > 1 and rows > 0 and stride[0] < (rows - 1) * ld + cols):
        raise ValueError("%s: columns have to lie next to each other, rows and matrices may not overlap, got strides %s" % (what, stride))
    return ws_matrix(t.data_ptr(), rows, cols, ld, code, batch, stride[0])


def _new_matrix(rows: int, cols: int, dtype: torch.dtype, device):
    """A new dense tensor and its descriptor."""
    t = torch.empty(rows, cols, dtype=dtype, device=device)
    return t, ws_matrix(t.data_ptr(), rows, cols, cols, _CODES[dtype], 1, 0)


def _index(t, what: str, n: int, device) -> int:
    if t is None:
        return 0
    _need(t, what, (torch.int32,), (1, 2), device)
    if t.numel() != n or not t.is_contiguous():
        raise ValueError("%s: expected %d contiguous int32, got %s" % (what, n, tuple(t.shape)))
    return t.data_ptr()


class Fp8Matrix:
    """rows x cols in 8 bits, or a batch of such matrices (weights of experts).

    ``codes`` ((batch x) rows x pitch, e4m3): columns padded with zero codes to a
    multiple of 16; rows may be further apart.  ``scales`` ((batch x) ceil(cols /
    128) x ceil(rows / block_rows), e8m0)."""

    __slots__ = ("codes", "scales", "rows", "cols", "block_rows", "_desc")

    def __init__(self, codes, scales, rows: int, cols: int, block_rows: int = 1):
        if block_rows not in (1, BLOCK):
            raise ValueError("block_rows is 1 or %d, got %r" % (BLOCK, block_rows))
        _need(codes, "codes", (E4M3,), (2, 3))
        _need(scales, "scales", (E8M0,), (codes.dim(),), codes.device)
        cs, ss, shape = codes.stride(), scales.stride(), codes.shape
        blocks, per = -(-cols // BLOCK), -(-rows // block_rows)
        batch = shape[0] if len(shape) == 3 else 1
        if shape[-2] != rows or not cols <= _up(cols, 16) <= shape[-1] or (shape[-1] > 1 and cs[-1] != 1):
            raise ValueError("codes %s of strides %s do not hold %d x %d values padded to 16 columns" % (tuple(shape), cs, rows, cols))
        if tuple(scales.shape) != tuple(shape[:-2]) + (blocks, per) or (per > 1 and ss[-1] != 1):
            raise ValueError("scales %s of strides %s: expected %s" % (tuple(scales.shape), ss, tuple(shape[:-2]) + (blocks, per)))
        ld = cs[-2] if rows > 1 and shape[-1] > 0 else _up(shape[-1], 16)
        if ld % 16 or codes.data_ptr() % 16 or (batch > 1 and cs[0] % 16):
            raise ValueError("codes: rows have to start at multiples of 16 bytes, got strides %s" % (cs,))
        ld_scales = ss[-2] if blocks > 1 else per
        if rows > 0 and cols > 0 and (ld < _up(cols, 16) or ld_scales < per or (batch > 1 and (
                cs[0] < (rows - 1) * ld + _up(cols, 16) or ss[0] < (blocks - 1) * ld_scales + per))):
            raise ValueError("rows and matrices may not overlap, got strides %s of codes and %s of scales" % (cs, ss))
        self.codes, self.scales, self.rows, self.cols, self.block_rows = codes, scales, rows, cols, block_rows
        self._desc = ws_fp8_matrix(codes.data_ptr(), scales.data_ptr(), rows, cols, ld,
                                   ld_scales, block_rows, batch,
                                   cs[0] if len(shape) == 3 else 0, ss[0] if len(shape) == 3 else 0)

    @property
    def batch(self):
        """Matrices of a batch, None for a single matrix."""
        return self.codes.shape[0] if self.codes.dim() == 3 else None

    @classmethod
    def empty(cls, rows: int, cols: int, block_rows: int = 1, batch: int | None = None, device="cuda"):
        if block_rows not in (1, BLOCK) or rows < 0 or cols < 0:
            raise ValueError("%d x %d with block_rows %r" % (rows, cols, block_rows))
        pitch, blocks, per = _up(cols, 16), -(-cols // BLOCK), -(-rows // block_rows)
        q = object.__new__(cls)
        if batch is None:
            q.codes = codes = torch.empty(rows, pitch, dtype=E4M3, device=device)
            q.scales = scales = torch.empty(blocks, per, dtype=E8M0, device=device)
        else:
            q.codes = codes = torch.empty(batch, rows, pitch, dtype=E4M3, device=device)
            q.scales = scales = torch.empty(batch, blocks, per, dtype=E8M0, device=device)
        q.rows, q.cols, q.block_rows = rows, cols, block_rows
        q._desc = ws_fp8_matrix(codes.data_ptr(), scales.data_ptr(), rows, cols, pitch, per, block_rows, 1 if batch is None else batch,
                                rows * pitch, blocks * per)
        return q

    def dequantize(self) -> torch.Tensor:
        """The values in binary32 (for tests and inspection; plain torch)."""
        s = self.scales.float().transpose(-1, -2).repeat_interleave(BLOCK, -1)[..., : self.cols]
        if self.block_rows > 1:
            s = s.repeat_interleave(self.block_rows, -2)[..., : self.rows, :]
        return self.codes[..., : self.cols].float() * s


def _fits(q, what: str, rows: int, cols: int, block_rows: int, batch, device) -> Fp8Matrix:
    if (q.rows, q.cols, q.block_rows, q.batch) != (rows, cols, block_rows, batch) or q.codes.device != device:
        raise ValueError("%s: expected %s x %d x %d with scales for %d rows on %s" % (what, batch, rows, cols, block_rows, device))
    return q


def _both(*qs):
    return [t for q in qs if q is not None for t in (q.codes, q.scales)]


def quantize_rows(x, index=None, out: Fp8Matrix | None = None, stream=None) -> Fp8Matrix:
    """x (rows x cols; f32, bf16 or f16) with a scale for every 1 x 128 values.
    index (int32): the source row of each result row; out of range, zeros."""
    m = _matrix(x, "x")
    if _elsewhere(x, stream):
        with _Call(x.device, stream, [x, index] + _both(out)):
            return quantize_rows(x, index, out)
    device = x.device
    rows = m.rows if index is None else index.numel()
    at = 0 if index is None else _index(index, "index", rows, device)
    q = Fp8Matrix.empty(rows, m.cols, device=device) if out is None else _fits(out, "out", rows, m.cols, 1, None, device)
    _check(_ws_fp8_quantize_rows(m, at, q._desc, _raw_stream(device.index)), "ws_fp8_quantize_rows")
    return q


def padded_rows(rows: int, groups: int) -> int:
    """Columns of the transposed form of ``rows`` rows in ``groups`` groups."""
    if not (0 <= rows <= _MOST and 0 <= groups <= _MOST):
        raise ValueError("padded_rows: %r rows in %r groups" % (rows, groups))
    return BLOCK * _lib.ws_fp8_padded_blocks(rows, groups)


def quantize_both(x, index=None, offsets=None, out=None, stream=None):
    """(rows, columns) of x from one read: quantize_rows' result, and that of the
    transpose.  With offsets (int32, groups + 1) the transpose's columns are those
    of each group, padded to 128 (see grouped_gradient), and rows in no group are
    zeros."""
    m = _matrix(x, "x")
    if _elsewhere(x, stream):
        with _Call(x.device, stream, [x, index, offsets] + _both(*(out or ()))):
            return quantize_both(x, index, offsets, out)
    device = x.device
    rows = m.rows if index is None else index.numel()
    at = _index(index, "index", rows, device)
    groups = 0 if offsets is None else offsets.numel() - 1
    if offsets is not None and groups < 1:
        raise ValueError("offsets: expected one more than groups")
    off = _index(offsets, "offsets", groups + 1, device)
    deep = padded_rows(rows, groups) if groups else rows
    if out is None:
        q, t = Fp8Matrix.empty(rows, m.cols, device=device), Fp8Matrix.empty(m.cols, deep, device=device)
    else:
        q, t = _fits(out[0], "out[0]", rows, m.cols, 1, None, device), _fits(out[1], "out[1]", m.cols, deep, 1, None, device)
    _check(_lib.ws_fp8_quantize_both(m, at, groups, off, q._desc, t._desc, _raw_stream(device.index)), "ws_fp8_quantize_both")
    return q, t


def quantize_weight(w, transposed: bool = True, out=None, stream=None):
    """(w, its transpose) with a scale for every 128 x 128 values; w is out x in,
    or experts x out x in.  transposed=False: (w, None)."""
    m = _matrix(w, "w", (2, 3))
    if _elsewhere(w, stream):
        with _Call(w.device, stream, [w] + _both(*(out or ()))):
            return quantize_weight(w, transposed, out)
    device = w.device
    batch = m.batch if w.dim() == 3 else None
    if out is None:
        q = Fp8Matrix.empty(m.rows, m.cols, BLOCK, batch, device)
        t = Fp8Matrix.empty(m.cols, m.rows, BLOCK, batch, device) if transposed else None
    else:
        q = _fits(out[0], "out[0]", m.rows, m.cols, BLOCK, batch, device)
        t = _fits(out[1], "out[1]", m.cols, m.rows, BLOCK, batch, device) if transposed else None
    _check(_lib.ws_fp8_quantize_weight(m, q._desc, t._desc if t is not None else None, _raw_stream(device.index)),
           "ws_fp8_quantize_weight")
    return q, t


def _result(C, out_dtype: str, shape, device):
    if C is None:
        dtype = _DTYPES.get(out_dtype)
        if dtype is None:
            raise ValueError("out_dtype is one of %s, got %r" % (sorted(_DTYPES), out_dtype))
        if len(shape) == 2:
            return _new_matrix(shape[0], shape[1], dtype, device)
        C = torch.empty(shape, dtype=dtype, device=device)
    elif tuple(C.shape) != tuple(shape):
        raise ValueError("C: expected %s, got %s" % (tuple(shape), tuple(C.shape)))
    return C, _matrix(C, "C", (len(shape),), device)


def _old(C0, beta: float, C):
    """Descriptor of what beta scales: C itself where no C0 is given."""
    if beta == 0.0:
        return None
    if C0 is None:
        raise ValueError("beta is not zero: C0 is needed")
    if C0.shape != C.shape or C0.dtype != C.dtype:
        raise ValueError("C0: expected %s %s, got %s %s" % (tuple(C.shape), C.dtype, tuple(C0.shape), C0.dtype))
    return _matrix(C0, "C0", (C.dim(),), C.device)


def plan(M: int, N: int, K: int, out_dtype: str = "bf16", groups: int = 0, depth: bool = False) -> list:
    """[(tile_m, tile_n, stages, rows, launch)]: the parts of product (groups 0), of
    grouped_product, or with depth of grouped_gradient over K rows."""
    out, n = (ws_fp8_kernel_info * 2)(), _i32(0)
    if out_dtype not in _DTYPES:
        raise ValueError("out_dtype is one of %s, got %r" % (sorted(_DTYPES), out_dtype))
    if not all(0 <= n <= _MOST for n in (M, N, K, groups)):
        raise _w.WsGemmError("ws_fp8_plan", _w.WS_ERR_INVALID_ARG)
    _check(_lib.ws_fp8_plan(M, N, K, _CODES[_DTYPES[out_dtype]], groups, int(depth), out, ctypes.byref(n)), "ws_fp8_plan")
    return [(k.tile_m, k.tile_n, k.stages, k.rows, k.launch) for k in out[: n.value]]


def product(A: Fp8Matrix, B: Fp8Matrix, C=None, out_dtype: str = "bf16", alpha: float = 1.0, beta: float = 0.0, C0=None,
            stream=None):
    """alpha A B^T + beta C0: A is M x K with scales for single rows, B is N x K with
    scales for 1 or 128 rows.  Written to C (M x N; its type counts) or a new
    tensor of out_dtype ("f32", "bf16", "f16").  C0 may be C.

    Results in 32 bits have binary32 sums.  Those in 16 bits come from the 8-bit
    matrix instruction at twice the rate, whose sums hold fewer bits: 1.5e-5 to
    5e-5 of the result before it is rounded (see ws_fp8.h); for binary32 sums in
    16 bits take out_dtype="f32" and round."""
    codes = A.codes
    if _elsewhere(codes, stream):
        with _Call(codes.device, stream, _both(A, B) + [C, C0]):
            return product(A, B, C, out_dtype, alpha, beta, C0)
    device = codes.device
    if codes.dim() == 3 or B.codes.dim() == 3 or B.codes.device != device:
        raise ValueError("A and B have to be single matrices on one device")
    if A.cols != B.cols or A.block_rows != 1:
        raise ValueError("A (%d x %d) and B (%d x %d) have to have as many columns, A scales for single rows" % (
            A.rows, A.cols, B.rows, B.cols))
    C, m = _result(C, out_dtype, (A.rows, B.rows), device)
    _check(_ws_fp8_product(A._desc, B._desc, alpha, beta, _old(C0, beta, C), m, _raw_stream(device.index)), "ws_fp8_product")
    return C


def grouped_product(A: Fp8Matrix, B: Fp8Matrix, offsets, C=None, out_dtype: str = "bf16", alpha: float = 1.0, stream=None):
    """Rows offsets[g] .. offsets[g + 1] - 1 of A times B[g]^T; rows in no group,
    before the first or after the last, become zeros.  offsets: int32 on the
    device, not decreasing.  Sums as in product."""
    device = A.codes.device
    if A.batch is not None or B.batch is None or A.cols != B.cols or A.block_rows != 1 or B.codes.device != device:
        raise ValueError("A has to be a single matrix with scales for single rows, B a batch of as many columns on its device")
    if _elsewhere(A.codes, stream):
        with _Call(device, stream, _both(A, B) + [offsets, C]):
            return grouped_product(A, B, offsets, C, out_dtype, alpha)
    off = _index(offsets, "offsets", B.batch + 1, device)
    C, m = _result(C, out_dtype, (A.rows, B.rows), device)
    _check(_lib.ws_fp8_grouped_product(A._desc, B._desc, B.batch, off, alpha, m, _raw_stream(device.index)), "ws_fp8_grouped_product")
    return C


def grouped_gradient(A: Fp8Matrix, B: Fp8Matrix, rows: int, offsets, C=None, out_dtype: str = "f32", alpha: float = 1.0,
                     beta: float = 0.0, C0=None, stream=None):
    """Weight gradient of grouped_product: for every group alpha A_g B_g^T + beta
    C0_g, contracted over the group's rows.  A (M x padded) and B (N x padded) are
    the columns that quantize_both makes of ``rows`` rows under these offsets; the
    result is groups x M x N, zeros (beta C0) for an empty group."""
    device = A.codes.device
    if _elsewhere(A.codes, stream):
        with _Call(device, stream, _both(A, B) + [offsets, C, C0]):
            return grouped_gradient(A, B, rows, offsets, C, out_dtype, alpha, beta, C0)
    groups = offsets.numel() - 1
    off = _index(offsets, "offsets", groups + 1, device)
    if A.batch is not None or B.batch is not None or A.block_rows != 1 or B.block_rows != 1 or B.codes.device != device:
        raise ValueError("A and B have to be single matrices with scales for single rows on one device")
    if groups < 1 or A.cols != B.cols or A.cols != padded_rows(rows, groups):
        raise ValueError("A and B have to hold the padded columns of %d rows in %d groups" % (rows, groups))
    C, m = _result(C, out_dtype, (groups, A.rows, B.rows), device)
    _check(_lib.ws_fp8_grouped_gradient(A._desc, B._desc, rows, groups, off, alpha, beta, _old(C0, beta, C), m,
                                        _raw_stream(device.index)), "ws_fp8_grouped_gradient")
    return C
