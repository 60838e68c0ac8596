"""Routing of tokens to experts and back over torch tensors (declared in
include/ws_experts.h; computed by the HIP kernels of libwsgemm.so).

    routes = sort(ids, experts)                    # ids: tokens x k
    xs = gather(x, routes)                         # rows by expert
    h = ...                                        # the experts' work on their rows
    y = combine(h, routes, weights)                # tokens x columns
    dh, dweights = combine_gradient(dy, h, routes, weights)
    dx = combine(dxs, routes)                      # gradient of gather

Streams and errors as in ``fp8``.  gather and combine are recorded by autograd
(once: their gradients are not differentiated again), so that the last two lines
are what their results' backward does; results in memory of the caller's (``out``)
cannot be, and ask for torch.no_grad() where an input requires a gradient.
"""
from __future__ import annotations

import ctypes

import torch
from torch.autograd.function import once_differentiable

from . import wsgemm as _w
from .fp8 import _Call, _check, _elsewhere, _matrix, _mp, _need, _new_matrix, _raw_stream

MAX_EXPERTS = 1024

_lib = _w.library()
_p, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
for _name, _args, _res in (
        ("ws_expert_sort_workspace", [_i64, _i32, _i32], _i64),
        ("ws_expert_sort", [_i64, _i32, _i32, _p, _i32, _p, _p, _p, _p, _i64, _p], _i32),
        ("ws_expert_gather", [_mp, _i32, _i32, _p, _p, _mp, _p], _i32),
        ("ws_expert_combine", [_mp, _i32, _p, _p, _mp, _p], _i32),
        ("ws_expert_combine_gradient", [_mp, _mp, _i32, _i32, _p, _p, _p, _mp, _p, _p], _i32)):
    getattr(_lib, _name).argtypes, getattr(_lib, _name).restype = _args, _res


class Routes:
    """Where every token's choices go: ``offsets`` (experts + 1), the ``token`` of
    each sorted row (-1: none) and the ``place`` of each choice (tokens x k; -1:
    none), int32 on the device."""

    __slots__ = ("offsets", "token", "place")

    def __init__(self, offsets, token, place):
        _need(offsets, "offsets", (torch.int32,), (1,))
        _need(token, "token", (torch.int32,), (1,), offsets.device)
        _need(place, "place", (torch.int32,), (2,), offsets.device)
        if offsets.numel() < 2 or token.numel() != place.numel() or not (
                offsets.is_contiguous() and token.is_contiguous() and place.is_contiguous()):
            raise ValueError("routes: offsets %s, token %s and place %s do not belong together" % (
                tuple(offsets.shape), tuple(token.shape), tuple(place.shape)))
        self.offsets, self.token, self.place = offsets, token, place

    @property
    def experts(self) -> int:
        return self.offsets.numel() - 1


def sort(ids, experts: int, stream=None) -> Routes:
    """Sorts the choices (tokens x k; int32 or int64; outside 0 .. experts - 1: none)
    by expert, each expert's in the order of the choices."""
    _need(ids, "ids", (torch.int32, torch.int64), (2,))
    if not ids.is_contiguous() or ids.shape[1] < 1:
        raise ValueError("ids: expected contiguous tokens x k, k at least 1, got %s of strides %s" % (tuple(ids.shape), ids.stride()))
    tokens, k = ids.shape
    need = _lib.ws_expert_sort_workspace(tokens, k, experts) if 0 < experts <= MAX_EXPERTS else -1
    if need < 0:
        raise ValueError("sort: 1 to %d experts, got %r, and at most 2^30 choices, got %d" % (MAX_EXPERTS, experts, ids.numel()))
    if _elsewhere(ids, stream):
        with _Call(ids.device, stream, [ids]):
            return sort(ids, experts)
    n, device = tokens * k, ids.device
    r = object.__new__(Routes)
    r.offsets = offsets = torch.empty(experts + 1, dtype=torch.int32, device=device)
    r.token = token = torch.empty(n, dtype=torch.int32, device=device)
    r.place = place = torch.empty(tokens, k, dtype=torch.int32, device=device)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _check(_lib.ws_expert_sort(tokens, k, experts, ids.data_ptr(), ids.element_size(), offsets.data_ptr(), token.data_ptr(),
                               place.data_ptr(), work.data_ptr() if need else 0, need, _raw_stream(device.index)), "ws_expert_sort")
    return r


def _out(out, what, rows, cols, like):
    """The result's tensor, new where none is given, and its descriptor."""
    if out is None:
        return _new_matrix(rows, cols, like.dtype, like.device)
    if tuple(out.shape) != (rows, cols) or out.dtype != like.dtype:
        raise ValueError("%s: expected %s %s, got %s %s" % (what, (rows, cols), like.dtype, tuple(out.shape), out.dtype))
    return out, _matrix(out, what, device=like.device)


def _weights(weights, routes):
    if weights is None:
        return 0
    _need(weights, "weights", (torch.float32,), (2,), routes.place.device)
    if weights.shape != routes.place.shape or not weights.is_contiguous():
        raise ValueError("weights: expected contiguous %s, got %s" % (tuple(routes.place.shape), tuple(weights.shape)))
    return weights.data_ptr()


def _recorded(out) -> bool:
    """Whether autograd has to know of a call on inputs that require a gradient."""
    if not torch.is_grad_enabled():
        return False
    if out is not None:
        raise ValueError("out: a result in the caller's memory is not recorded for gradients; call it under torch.no_grad()")
    return True


class _Gather(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, routes):
        ctx.save_for_backward(routes.offsets, routes.token, routes.place)
        return gather(x, routes)

    @staticmethod
    @once_differentiable
    def backward(ctx, dxs):
        return combine(dxs.contiguous(), Routes(*ctx.saved_tensors)), None


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h, weights, routes):
        of_weights = ctx.needs_input_grad[1]
        ctx.save_for_backward(h if of_weights else None, weights, routes.offsets, routes.token, routes.place)
        return combine(h, routes, weights)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        h, weights, *routes = ctx.saved_tensors
        dh, dweights = _gradient(dy.contiguous(), h, Routes(*routes), weights, None, ctx.needs_input_grad[1])
        return dh if ctx.needs_input_grad[0] else None, dweights, None


def gather(x, routes: Routes, out=None, stream=None):
    """x (tokens x columns; f32, bf16 or f16) by sorted row; zeros for rows of no token."""
    m = _matrix(x, "x", device=routes.token.device)
    tokens, k = routes.place.shape
    if m.rows != tokens:
        raise ValueError("x: %d rows for %d tokens" % (m.rows, tokens))
    if _elsewhere(x, stream):
        with _Call(x.device, stream, [x, routes.offsets, routes.place, out]):
            return gather(x, routes, out)
    if x.requires_grad and _recorded(out):
        return _Gather.apply(x, routes)
    out, mo = _out(out, "out", routes.token.numel(), m.cols, x)
    _check(_lib.ws_expert_gather(m, k, routes.experts, routes.offsets.data_ptr(), routes.place.data_ptr(), mo,
                                 _raw_stream(x.get_device())), "ws_expert_gather")
    return out


def combine(h, routes: Routes, weights=None, out=None, stream=None):
    """Each token's sum of its choices' rows of h, times weights (tokens x k, f32)
    where given; summed in binary32.  A token without a place gets zeros."""
    m = _matrix(h, "h", device=routes.token.device)
    if m.rows != routes.token.numel():
        raise ValueError("h: %d rows for %d choices" % (m.rows, routes.token.numel()))
    w, (tokens, k) = _weights(weights, routes), routes.place.shape
    if _elsewhere(h, stream):
        with _Call(h.device, stream, [h, routes.place, weights, out]):
            return combine(h, routes, weights, out)
    if (h.requires_grad or (weights is not None and weights.requires_grad)) and _recorded(out):
        return _Combine.apply(h, weights, routes)
    out, mo = _out(out, "out", tokens, m.cols, h)
    _check(_lib.ws_expert_combine(m, k, routes.place.data_ptr(), w, mo, _raw_stream(h.get_device())), "ws_expert_combine")
    return out


def combine_gradient(dy, h, routes: Routes, weights=None, dh=None, stream=None):
    """(dh, dweights) of combine: dh like h, rows without a token zero; dweights
    tokens x k in binary32, None where weights is None (then h may be None).  Not
    recorded by autograd."""
    return _gradient(dy, h, routes, weights, dh, weights is not None, stream)


def _gradient(dy, h, routes, weights, dh, of_weights, stream=None):
    """of_weights: dweights is wanted (else None, and h is not looked at)."""
    m = _matrix(dy, "dy", device=routes.token.device)
    w, (tokens, k) = _weights(weights, routes), routes.place.shape
    if m.rows != tokens:
        raise ValueError("dy: %d rows for %d tokens" % (m.rows, tokens))
    if of_weights:
        mh = _matrix(h, "h", device=dy.device)
        if (mh.rows, mh.cols) != (routes.token.numel(), m.cols) or h.dtype != dy.dtype:
            raise ValueError("h: expected %s %s, got %s %s" % ((routes.token.numel(), m.cols), dy.dtype, tuple(h.shape), h.dtype))
    else:
        mh = None
    if _elsewhere(dy, stream):
        with _Call(dy.device, stream, [dy, h, routes.offsets, routes.place, weights, dh]):
            return _gradient(dy, h, routes, weights, dh, of_weights)
    dh, mdh = _out(dh, "dh", routes.token.numel(), m.cols, dy)
    dw = torch.empty(tokens, k, dtype=torch.float32, device=dy.device) if of_weights else None
    _check(_lib.ws_expert_combine_gradient(m, mh, k, routes.experts, routes.offsets.data_ptr(), routes.place.data_ptr(), w, mdh,
                                           dw.data_ptr() if dw is not None else 0, _raw_stream(dy.get_device())),
           "ws_expert_combine_gradient")
    return dh, dw
