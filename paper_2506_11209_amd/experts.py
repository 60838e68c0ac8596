"""Routing of tokens to experts and back over torch tensors (declared in
include/ws_experts.h; computed by the HIP kernels of libwsgemm.so).

    weights, ids, counts, loss = choose(logits, k) # logits: tokens x experts
    routes = sort(ids, experts)                    # ids: tokens x k
    xs = gather(x, routes)                         # rows by expert
    h = ...                                        # the experts' work on their rows
    y = combine(h, routes, weights)                # tokens x columns
    dh, dweights = combine_gradient(dy, h, routes, weights)
    dx = combine(dxs, routes)                      # gradient of gather
    dlogits = choose_gradient(dweights, dloss, logits, weights, ids, counts)

Streams and errors as in ``fp8``.  choose, gather and combine are recorded by
autograd (once: their gradients are not differentiated again), so that the last
three lines are what their results' backward does; results in memory of the
caller's (``out``) cannot be, and ask for torch.no_grad() where an input requires a
gradient.  Forward mode is refused (NotImplementedError).
"""
from __future__ import annotations

import ctypes

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import wsgemm as _w
from .fp8 import _Call, _check, _elsewhere, _matrix, _mp, _need, _new_matrix, _raw_stream

MAX_EXPERTS = 1024
MAX_CHOICES = 32

_lib = _w.library()
_p, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
for _name, _args, _res in (
        ("ws_expert_choose_workspace", [_i64, _i32, _i32], _i64),
        ("ws_expert_choose", [_mp, _i32, _p, _p, _p, _p, _p, _i64, _p], _i32),
        ("ws_expert_choose_gradient", [_mp, _i32, _p, _p, _p, _p, _p, _mp, _p], _i32),
        ("ws_expert_sort_workspace", [_i64, _i32, _i32], _i64),
        ("ws_expert_sort", [_i64, _i32, _i32, _p, _i32, _p, _p, _p, _p, _i64, _p], _i32),
        ("ws_expert_gather", [_mp, _i32, _i32, _p, _p, _mp, _p], _i32),
        ("ws_expert_combine", [_mp, _i32, _p, _p, _mp, _p], _i32),
        ("ws_expert_combine_gradient", [_mp, _mp, _i32, _i32, _p, _p, _p, _mp, _p, _p], _i32)):
    getattr(_lib, _name).argtypes, getattr(_lib, _name).restype = _args, _res


def _no_forward_mode(what, *tensors):
    """Refuses inputs with a tangent, which the kernels would drop."""
    if forward_ad._current_level >= 0 and any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise NotImplementedError("%s: not differentiated in forward mode" % what)


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


class _Choose(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, k):
        weights, ids, counts, loss = choose(logits, k)
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(ids, counts)
        ctx.save_for_backward(logits, weights, ids, counts)
        return weights, ids, counts, loss

    @staticmethod
    @once_differentiable
    def backward(ctx, dweights, _ids, _counts, dloss):
        if dweights is None and dloss is None:
            return None, None
        if dweights is not None:
            dweights = dweights.contiguous()
        return choose_gradient(dweights, dloss, *ctx.saved_tensors), None


def _logits(logits):
    m = _matrix(logits, "logits")
    if m.cols > MAX_EXPERTS:
        raise ValueError("logits: at most %d experts, got %d" % (MAX_EXPERTS, m.cols))
    return m


def _dense(t, what, dtype, shape, device):
    """Refuses all but a contiguous tensor of this type and shape."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        _need(t, what, (dtype,), (len(shape),), device)
        raise ValueError("%s: expected contiguous %s, got %s of strides %s" % (what, tuple(shape), tuple(t.shape), t.stride()))


def choose(logits, k: int, stream=None):
    """(weights, ids, counts, loss) of a router's logits (tokens x experts; f32, bf16
    or f16).  ids (tokens x k, int32): each token's k largest logits, the largest
    first, the lowest index first among equals; -inf is not chosen, -1 stands where
    none is left (a masked token is a row of -inf).  weights (tokens x k, f32): the
    softmax over a token's choices.  counts (experts + 1, int32): the choices of each
    expert, and at last the tokens that have any.  loss (f32, no dimensions): experts
    * sum over the experts of their share of the choices * the mean of their softmax
    probability over the tokens with a choice.  Gradients flow from weights and loss."""
    m = _logits(logits)
    tokens, experts = m.rows, m.cols
    need = _lib.ws_expert_choose_workspace(tokens, experts, k) if 0 < k <= min(experts, MAX_CHOICES) else -1
    if need < 0:
        raise ValueError("choose: 1 to %d of the %d experts and at most 2^30 choices, got k = %r for %d tokens" % (
            MAX_CHOICES, experts, k, tokens))
    _no_forward_mode("choose", logits)
    if _elsewhere(logits, stream):
        with _Call(logits.device, stream, [logits]):
            return choose(logits, k)
    if logits.requires_grad and torch.is_grad_enabled():
        return _Choose.apply(logits, k)
    device = logits.device
    weights = torch.empty(tokens, k, dtype=torch.float32, device=device)
    ids = torch.empty(tokens, k, dtype=torch.int32, device=device)
    counts = torch.empty(experts + 1, dtype=torch.int32, device=device)
    loss = torch.empty((), dtype=torch.float32, device=device)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _check(_lib.ws_expert_choose(m, k, weights.data_ptr(), ids.data_ptr(), counts.data_ptr(), loss.data_ptr(),
                                 work.data_ptr() if need else 0, need, _raw_stream(device.index)), "ws_expert_choose")
    return weights, ids, counts, loss


def choose_gradient(dweights, dloss, logits, weights, ids, counts, out=None, stream=None):
    """dlogits (like logits) of choose, from the gradients of its weights (tokens x k)
    and its loss (one value); each may be None, which is zero.  logits and the rest as
    choose took and gave them; an id out of range counts as none.  Not recorded by
    autograd."""
    m = _logits(logits)
    device = logits.device
    _need(ids, "ids", (torch.int32,), (2,), device)
    tokens, k = shape = ids.shape
    if tokens != m.rows or not 0 < k <= min(m.cols, MAX_CHOICES) or not ids.is_contiguous():
        raise ValueError("ids: expected contiguous %d x k, k up to %d, got %s" % (m.rows, min(m.cols, MAX_CHOICES), tuple(shape)))
    _dense(weights, "weights", torch.float32, shape, device)
    if dweights is not None:
        _dense(dweights, "dweights", torch.float32, shape, device)
    _dense(counts, "counts", torch.int32, (m.cols + 1,), device)
    if dloss is not None:
        _need(dloss, "dloss", (torch.float32,), (0, 1), device)
        if dloss.numel() != 1:
            raise ValueError("dloss: expected one value, got %s" % (tuple(dloss.shape),))
    if _elsewhere(logits, stream):
        with _Call(device, stream, [dweights, dloss, logits, weights, ids, counts, out]):
            return choose_gradient(dweights, dloss, logits, weights, ids, counts, out)
    out, mo = _out(out, "out", m.rows, m.cols, logits)
    _check(_lib.ws_expert_choose_gradient(m, k, dweights.data_ptr() if dweights is not None else 0,
                                          dloss.data_ptr() if dloss is not None else 0, weights.data_ptr(), ids.data_ptr(),
                                          counts.data_ptr(), mo, _raw_stream(device.index)), "ws_expert_choose_gradient")
    return out


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
    _no_forward_mode("gather", x)
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
    _no_forward_mode("combine", h, weights)
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
