"""The gradients of a linear layer in 8 bits along directions in which the loss
changes, so that a gradient that is zero, of the wrong sign or scale is far out."""
import numpy as np
import pytest
import torch

from tests import fp8_ref as ref
from tests.gpu_helpers import log

# A code is within 2^-4 of its value, evenly spread over that at the most: 2^-4 / sqrt(3) = 3.6 % in
# the mean square; two factors with independent errors 5.1 % of the root of the terms' squares, which
# is what the norm of a product of random matrices is.  Its scatter over T = 200 terms and 10^4
# elements is below a hundredth of that; values below a block's least normal code add less than 2^-9 /
# 448 of the block's largest each.
TOLERANCE = 0.06


def difference(loss, at, along, h=2.0 ** -10):
    return (loss(at + h * along) - loss(at - h * along)) / (2 * h)


def accepted(got, exact, loss, at):
    """got against the exact gradient in norm, and against the loss's difference along it."""
    d = difference(loss, at, exact)
    return np.linalg.norm(got - exact) <= TOLERANCE * np.linalg.norm(exact) and abs((got * exact).sum() - d) <= TOLERANCE * abs(d)


def problem():
    g = np.random.default_rng(0)
    x, w, dy = g.standard_normal((200, 264)), g.standard_normal((136, 264)), g.standard_normal((200, 136))
    x, w, dy = (v.astype(np.float32).astype(np.float64) for v in (x, w, dy))
    return x, w, dy, lambda m: (dy * (x @ m.T)).sum(), lambda m: (dy * (m @ w.T)).sum()


def quantized(v, block_rows=1):
    codes, scales = ref.quantize(v, block_rows)
    s = np.repeat(scales.T, 128, axis=1)
    return (codes * np.repeat(s, block_rows, axis=0)[: len(codes), : codes.shape[1]])[:, : v.shape[1]]


def test_the_check_tells_right_from_wrong():
    """On the CPU, with the definition's quantisation."""
    x, w, dy, of_w, of_x = problem()
    for got, exact, loss, at in ((quantized(dy.T) @ quantized(x.T).T, dy.T @ x, of_w, w),
                                 (quantized(dy) @ quantized(w.T, 128).T, dy @ w, of_x, x)):
        assert accepted(got, exact, loss, at)
        for wrong in (0 * got, -got, 1.1 * got, 0.9 * got, np.roll(got, 1, 0), got * (np.arange(got.shape[1]) % 50 != 7)):
            assert not accepted(wrong, exact, loss, at)


@pytest.mark.gpu
def test_linear_layer():
    fp8 = pytest.importorskip("paper_2506_11209_amd.fp8")
    log("case gradient directions")
    x, w, dy, of_w, of_x = problem()
    cuda = lambda v: torch.from_numpy(v).float().cuda()  # noqa: E731
    (_, xt), (_, wt), (gq, gt) = fp8.quantize_both(cuda(x)), fp8.quantize_weight(cuda(w)), fp8.quantize_both(cuda(dy))
    for out in ("f32", "bf16"):
        assert accepted(ref.f64(fp8.product(gt, xt, out_dtype=out)), dy.T @ x, of_w, w)
        assert accepted(ref.f64(fp8.product(gq, wt, out_dtype=out)), dy @ w, of_x, x)


@pytest.mark.gpu
def test_groups():
    """Each group's weight gradient, and the input gradient, of a grouped layer."""
    fp8 = pytest.importorskip("paper_2506_11209_amd.fp8")
    log("case gradient directions of groups")
    offsets, (x, _, dy, _, _) = [0, 90, 90, 200], problem()
    w = np.random.default_rng(1).standard_normal((3, 136, 264)).astype(np.float32).astype(np.float64)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    cuda = lambda v: torch.from_numpy(v).float().cuda()  # noqa: E731
    (_, xt), (_, wt), (gq, gt) = fp8.quantize_both(cuda(x), offsets=off), fp8.quantize_weight(cuda(w)), fp8.quantize_both(cuda(dy), offsets=off)
    dw, dx = ref.f64(fp8.grouped_gradient(gt, xt, 200, off)), ref.f64(fp8.grouped_product(gq, wt, off, out_dtype="f32"))
    assert (dw[1] == 0).all()
    for g, (lo, hi) in enumerate(ref.segments(offsets, 200)):
        if hi > lo:
            a, b = x[lo:hi], dy[lo:hi]
            assert accepted(dw[g], b.T @ a, lambda m: (b * (a @ m.T)).sum(), w[g])
            assert accepted(dx[lo:hi], b @ w[g], lambda m: (b * (m @ w[g].T)).sum(), a)
