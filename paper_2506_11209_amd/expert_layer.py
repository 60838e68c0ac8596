"""A layer of experts in 8 bits, trained and served with this library's operators.

Every token goes to k of E experts, y = sum over its choices of weight * W2 silu(W1
x).  Forward: the choices are sorted by expert, the tokens' rows are quantised in
that order (gathered on the way, both forms from one read), and the experts'
products run as grouped products; the rows go back to their tokens with the
router's weights.  Backward: the gradient of the way back, the input gradients as
grouped products with the transposed weights, the weight gradients as products
over each expert's rows in 32 bits.

    python -m paper_2506_11209_amd.expert_layer [--tokens 4096] [--experts 16] ...

times a training step and a decoding step on the GPU and prints a line for each.
"""
from __future__ import annotations

import argparse
import json
import time

import torch
from torch.autograd.function import once_differentiable

from . import experts, fp8


class _Experts(torch.autograd.Function):
    """y of x, the choices' weights (tokens x k, f32) and ids (tokens x k); w1 is E x
    hidden x columns, w2 is E x columns x hidden.  Only what the gradients that are
    asked for need is quantised, kept and computed."""

    @staticmethod
    def forward(ctx, x, weights, w1, w2, ids):
        of_x, of_weights, of_w1, of_w2, _ = ctx.needs_input_grad
        of_h = of_x or of_w1  # of the first product
        routes = experts.sort(ids, w1.shape[0])
        xq, xt = _operand(x, routes, of_w1, index=routes.token)
        w1q, w1t = fp8.quantize_weight(w1, transposed=of_x)
        h = fp8.grouped_product(xq, w1q, routes.offsets)
        aq, at = _operand(torch.nn.functional.silu(h), routes, of_w2)
        w2q, w2t = fp8.quantize_weight(w2, transposed=of_h)
        rows = fp8.grouped_product(aq, w2q, routes.offsets)
        y = experts.combine(rows, routes, weights)
        # quantised operands are kept, not the tensors they came from
        operands = (xt, at, w1t, w2t)
        ctx.shapes = [q and (q.rows, q.cols, q.block_rows) for q in operands]
        ctx.save_for_backward(weights, h if of_h else None, rows if of_weights else None, routes.offsets, routes.token, routes.place,
                              *(t for q in operands for t in ((q.codes, q.scales) if q else (None, None))))
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        of_x, of_weights, of_w1, of_w2, _ = ctx.needs_input_grad
        weights, h, rows, off, token, place, *kept = ctx.saved_tensors
        xt, at, w1t, w2t = (s and fp8.Fp8Matrix(*kept[2 * i:2 * i + 2], *s) for i, s in enumerate(ctx.shapes))
        routes, n = experts.Routes(off, token, place), token.numel()
        dx = dw1 = dw2 = None
        drows, dweights = experts._gradient(dy.contiguous(), rows, routes, weights, None, of_weights)
        if of_x or of_w1 or of_w2:
            gq, gt = _operand(drows, routes, of_w2)
        if of_w2:
            dw2 = fp8.grouped_gradient(gt, at, n, off)
        if of_x or of_w1:
            da = fp8.grouped_product(gq, w2t, off).float()
            s = torch.sigmoid(h.float())
            dh = (da * (s * (1.0 + h.float() * (1.0 - s)))).to(h.dtype)
            hq, ht = _operand(dh, routes, of_w1)
        if of_w1:
            dw1 = fp8.grouped_gradient(ht, xt, n, off)
        if of_x:
            dx = experts.combine(fp8.grouped_product(hq, w1t, off), routes)
        return dx, dweights, dw1, dw2, None


def _operand(x, routes, columns: bool, index=None):
    """x, one row for each choice, for a grouped product, and its columns where a
    weight gradient contracts over them."""
    if columns:
        return fp8.quantize_both(x, index=index, offsets=routes.offsets)
    return fp8.quantize_rows(x, index=index), None


class ExpertLayer(torch.nn.Module):
    """columns -> hidden -> columns by k of `count` experts; master weights in
    binary32, activations in bf16."""

    def __init__(self, columns: int, hidden: int, count: int, k: int, device="cuda", generator=None):
        super().__init__()
        make = lambda *s: torch.nn.Parameter(  # noqa: E731
            torch.randn(*s, device=device, generator=generator) / s[-1] ** 0.5)
        self.router, self.w1, self.w2 = make(count, columns), make(count, hidden, columns), make(count, columns, hidden)
        self.k = k

    def route(self, x):
        """(weights, ids) of each token's k best experts."""
        score, ids = (x.float() @ self.router.t()).topk(self.k, dim=1)
        return score.softmax(1), ids

    def forward(self, x):
        weights, ids = self.route(x)
        return _Experts.apply(x, weights, self.w1, self.w2, ids)

    @torch.no_grad()
    def serving_weights(self):
        """The experts' weights in 8 bits, laid out once for serve."""
        return fp8.quantize_weight(self.w1, transposed=False)[0], fp8.quantize_weight(self.w2, transposed=False)[0]

    @torch.no_grad()
    def serve(self, x, quantized):
        """forward without what training keeps; quantized: serving_weights()."""
        weights, ids = self.route(x)
        routes = experts.sort(ids, self.w1.shape[0])
        h = fp8.grouped_product(fp8.quantize_rows(x, index=routes.token), quantized[0], routes.offsets)
        rows = fp8.grouped_product(fp8.quantize_rows(torch.nn.functional.silu(h)), quantized[1], routes.offsets)
        return experts.combine(rows, routes, weights)


def _time(step, steps: int) -> float:
    for _ in range(3):
        step()
    torch.cuda.synchronize()
    begin = time.perf_counter()
    for _ in range(steps):
        step()
    torch.cuda.synchronize()
    return (time.perf_counter() - begin) / steps


def main(argv=None) -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("tokens", 4096), ("decode", 32), ("columns", 2048), ("hidden", 4096), ("experts", 16), ("k", 2), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(0)
    layer = ExpertLayer(a.columns, a.hidden, a.experts, a.k, generator=g)
    x = torch.randn(a.tokens, a.columns, device="cuda", generator=g).bfloat16().requires_grad_()
    dy = torch.randn(a.tokens, a.columns, device="cuda", generator=g).bfloat16()
    few = x.detach()[: a.decode].contiguous()
    quantized = layer.serving_weights()

    def train():
        layer.zero_grad()
        x.grad = None
        layer(x).backward(dy)

    flops = 6.0 * a.tokens * a.k * a.columns * a.hidden * 2
    s = _time(train, a.steps)
    print(json.dumps({"step": "training", "tokens": a.tokens, "us": round(s * 1e6, 1), "tflops": round(flops / s / 1e12, 1)}), flush=True)
    s = _time(lambda: layer.serve(few, quantized), a.steps)
    print(json.dumps({"step": "decoding", "tokens": few.shape[0], "us": round(s * 1e6, 1)}), flush=True)


if __name__ == "__main__":
    main()
