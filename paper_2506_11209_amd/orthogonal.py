"""Orthogonalised updates over torch tensors (declared in include/ws_orthogonal.h;
computed by the HIP kernels of libwsgemm.so, with no other path).

    u = orthogonalize(grad)                       # (batch x) rows x columns -> bf16
    optimizer = OrthogonalMomentum(layer.parameters(), lr=0.02)

Streams and errors as in ``fp8``; nothing here is recorded by autograd.
"""
from __future__ import annotations

import ctypes

import torch

from . import wsgemm as _w
from .fp8 import _Call, _check, _elsewhere, _matrix, _mp, _raw_stream, ws_matrix, _CODES

MAX_STEPS = 100

_lib = _w.library()
_p, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
for _name, _args, _res in (("ws_orthogonal_workspace", [_i64, _i64, _i32], _i64),
                           ("ws_orthogonalize", [_mp, _i32, _mp, _p, _i64, _p], _i32)):
    getattr(_lib, _name).argtypes, getattr(_lib, _name).restype = _args, _res


def _counts(steps) -> bool:
    return isinstance(steps, int) and 1 <= steps <= MAX_STEPS


def _need_bytes(rows: int, cols: int, batch: int, what: str) -> int:
    """Work memory for a batch of matrices; refuses sizes that no launch holds."""
    need = _lib.ws_orthogonal_workspace(rows, cols, batch) if max(rows, cols, batch) < 1 << 31 else -1
    if need < 0:
        raise ValueError("%s: sizes %s are too large" % (what, (batch, rows, cols)))
    return need


def orthogonalize(G, steps: int = 5, out=None, stream=None):
    """G (rows x columns, or a batch of such matrices; f32, bf16 or f16) with its
    singular values brought near 1 by ``steps`` Newton-Schulz steps, in bf16: X = G /
    |G|, then X <- a X + (b A + c A^2) X with A = X X^T.  Each matrix of a batch for
    itself; zeros stay zeros, a matrix with an infinity or NaN becomes NaN.  out may not
    overlap G."""
    m = _matrix(G, "G", (2, 3))
    if not _counts(steps):
        raise ValueError("steps: 1 to %d, got %r" % (MAX_STEPS, steps))
    need = _need_bytes(m.rows, m.cols, m.batch, "orthogonalize")
    if out is not None and (out.shape != G.shape or out.dtype != torch.bfloat16):
        raise ValueError("out: expected %s bf16, got %s %s" % (tuple(G.shape), tuple(out.shape), out.dtype))
    if _elsewhere(G, stream):
        with _Call(G.device, stream, [G, out]):
            return orthogonalize(G, steps, out)
    device = G.device
    if out is None:
        out = torch.empty(G.shape, dtype=torch.bfloat16, device=device)
        mo = ws_matrix(out.data_ptr(), m.rows, m.cols, m.cols, _CODES[torch.bfloat16], m.batch, m.rows * m.cols)
    else:
        mo = _matrix(out, "out", (G.dim(),), device)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _check(_lib.ws_orthogonalize(m, steps, mo, work.data_ptr() if need else 0, need, _raw_stream(device.index)), "ws_orthogonalize")
    return out


class OrthogonalMomentum(torch.optim.Optimizer):
    """Momentum whose updates are orthogonalised: for matrices and batches of them (the
    weights of experts), b <- momentum b + g, u = g + momentum b (or b, without nesterov),
    w <- (1 - lr weight_decay) w - lr max(1, rows / columns)^0.5 orthogonalize(u).
    b is kept in binary32 whatever the parameters' type.  Sizes and options are checked when
    a group is added, and all gradients before a step changes anything."""

    def __init__(self, params, lr: float = 0.02, momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0, steps: int = 5):
        defaults = dict(lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=weight_decay, steps=steps)
        self._check_options(defaults)
        super().__init__(params, defaults)

    @staticmethod
    def _check_options(group):
        lr, momentum, weight_decay, steps = (group[k] for k in ("lr", "momentum", "weight_decay", "steps"))
        if not lr >= 0 or not 0 <= momentum < 1 or not weight_decay >= 0 or not _counts(steps):
            raise ValueError("lr %r, momentum %r, weight_decay %r, steps %r" % (lr, momentum, weight_decay, steps))

    def add_param_group(self, param_group):
        super().add_param_group(param_group)
        group = self.param_groups[-1]
        try:
            self._check_options(group)
            for p in group["params"]:
                if p.dim() not in (2, 3):
                    raise ValueError("parameters have to be matrices or batches of them, got %s" % (tuple(p.shape),))
                _need_bytes(p.shape[-2], p.shape[-1], p.shape[0] if p.dim() == 3 else 1, "parameter")
        except ValueError:
            del self.param_groups[-1]
            raise

    def load_state_dict(self, state_dict):
        super().load_state_dict(state_dict)  # which rounds to the parameters' type
        own = [p for group in self.param_groups for p in group["params"]]
        for p, i in zip(own, (i for group in state_dict["param_groups"] for i in group["params"])):
            if i in state_dict["state"]:
                self.state[p]["momentum"] = state_dict["state"][i]["momentum"].to(p.device, torch.float32, copy=True)

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for group in self.param_groups:  # all of it before the first change
            self._check_options(group)
            for p in group["params"]:
                if p.grad is not None and (p.grad.layout != torch.strided or not p.grad.is_cuda or p.grad.dtype not in _CODES):
                    raise ValueError("gradients have to be dense cuda tensors of f32, bf16 or f16, got %s of %s on %s" % (
                        p.grad.layout, p.grad.dtype, p.grad.device))
        for group in self.param_groups:
            for p in group["params"]:
                if p.grad is None:
                    continue
                state, momentum = self.state[p], group["momentum"]
                if "momentum" not in state:
                    state["momentum"] = torch.zeros_like(p, dtype=torch.float32, memory_format=torch.contiguous_format)
                b = state["momentum"]
                b.mul_(momentum).add_(p.grad)
                u = torch.add(p.grad, b, alpha=momentum) if group["nesterov"] else b
                u = orthogonalize(u.contiguous(), group["steps"])
                if group["weight_decay"]:
                    p.mul_(1 - group["lr"] * group["weight_decay"])
                p.add_(u, alpha=-group["lr"] * max(1.0, p.shape[-2] / max(1, p.shape[-1])) ** 0.5)
        return loss
