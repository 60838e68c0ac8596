"""The layer of experts against its own steps in 64 bits: the same quantisation and
the same roundings between them, so that what is left is how sums round."""
import numpy as np
import pytest
import torch

from tests import fp8_ref as ref
from tests.gpu_helpers import log

# What differs from the layer's own arithmetic: sums (6e-5 of a result in 16 bits at the most on such
# values) that move at most one in 60 of the 16-bit values between to a neighbour, 2^-8 away; one in
# sixteen of those then moves a code, by 2^-3 of its value: sqrt(1 / 960) / 8 = 0.4 %.  Three such steps
# follow one another: 0.7 %; and one in a hundred blocks may take another scale, which its codes
# hardly show.  A missing factor or term shows with 5 % and more.
TOLERANCE = 0.02


def bf16(v):
    return torch.from_numpy(np.ascontiguousarray(v)).to(torch.bfloat16).double().numpy()


def rows_of(v, block_rows=1):
    """v after quantisation in blocks of block_rows x 128."""
    if v.size == 0:
        return v
    codes, scales = ref.quantize(v, block_rows)
    s = np.repeat(scales.T, 128, axis=1)
    return (codes * np.repeat(s, block_rows, axis=0)[: len(codes), : codes.shape[1]])[:, : v.shape[1]]


def columns_of(v):
    return rows_of(v.T).T


def slope_of_silu(h):
    s = 1.0 / (1.0 + np.exp(-h))
    return s * (1.0 + h * (1.0 - s))


def steps(x, w1, w2, weights, ids, dy, slope=slope_of_silu):
    """(y, dx, dweights, dw1, dw2) of the layer's formula, step by step."""
    y, dx = np.zeros_like(x), np.zeros_like(x)
    dweights, dw1, dw2 = np.zeros_like(weights), np.zeros_like(w1), np.zeros_like(w2)
    for e in range(len(w1)):
        t, j = np.nonzero(ids == e)  # by token, then by choice
        if not len(t):
            continue
        q1, q2, xe = rows_of(w1[e], 128), rows_of(w2[e], 128), x[t]
        h = bf16(rows_of(xe) @ q1.T)
        a = bf16(h / (1.0 + np.exp(-h)))
        rows = bf16(rows_of(a) @ q2.T)
        np.add.at(y, t, weights[t, j][:, None] * rows)
        dweights[t, j] = (dy[t] * rows).sum(1)
        drows = bf16(weights[t, j][:, None] * dy[t])
        dw2[e] = columns_of(drows).T @ columns_of(a)
        da = bf16(rows_of(drows) @ q2)
        dh = bf16(da * slope(h))
        dw1[e] = columns_of(dh).T @ columns_of(xe)
        np.add.at(dx, t, bf16(rows_of(dh) @ q1))
    return y, dx, dweights, dw1, dw2


def off(a, b):
    return np.linalg.norm(a - b) / np.linalg.norm(b)


def problem(T, columns, hidden, E, k):
    g = np.random.default_rng(T)
    x, dy = bf16(g.standard_normal((T, columns))), bf16(g.standard_normal((T, columns)))
    w1 = (g.standard_normal((E, hidden, columns)) / columns ** 0.5).astype(np.float32).astype(np.float64)
    w2 = (g.standard_normal((E, columns, hidden)) / hidden ** 0.5).astype(np.float32).astype(np.float64)
    weights = g.dirichlet(np.ones(k), T).astype(np.float32).astype(np.float64)
    ids = np.argsort(g.standard_normal((T, E)), axis=1)[:, :k]
    ids[T // 2] = -1  # a token without experts
    return x, w1, w2, weights, ids, dy


CASES = [(200, 256, 384, 8, 2), (33, 136, 200, 5, 3), (300, 130, 120, 3, 1)]


@pytest.mark.parametrize("case", CASES)
def test_the_tolerance_tells_wrong_steps(case):
    """On the CPU: silu's slope without its second term, or with another sign there, is out."""
    p = problem(*case)
    right = steps(*p)
    for wrong in (lambda h: 1.0 / (1.0 + np.exp(-h)), lambda h: 1.0 / (1.0 + np.exp(-h)) * (1.0 - h / (1.0 + np.exp(h))),
                  lambda h: 1.05 * slope_of_silu(h)):
        got = steps(*p, slope=wrong)
        assert off(got[1], right[1]) > 2 * TOLERANCE and off(got[3], right[3]) > 2 * TOLERANCE


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES)
def test_layer(case):
    expert_layer = pytest.importorskip("paper_2506_11209_amd.expert_layer")
    log("case layer steps %s" % (case,))
    x, w1, w2, weights, ids, dy = problem(*case)
    cuda = lambda v, t: torch.from_numpy(v).to(t).cuda().requires_grad_()  # noqa: E731
    xd, wd = cuda(x, torch.bfloat16), cuda(weights, torch.float32)
    w1d, w2d = cuda(w1, torch.float32), cuda(w2, torch.float32)
    y = expert_layer._Experts.apply(xd, wd, w1d, w2d, torch.from_numpy(ids).cuda())
    y.backward(torch.from_numpy(dy).to(torch.bfloat16).cuda())
    for name, got, want in zip(("y", "dx", "dweights", "dw1", "dw2"), (y, xd.grad, wd.grad, w1d.grad, w2d.grad),
                               steps(x, w1, w2, weights, ids, dy)):
        assert off(ref.f64(got), want) <= TOLERANCE, name
    gone = len(x) // 2
    assert (y[gone] == 0).all() and (xd.grad[gone] == 0).all() and (wd.grad[gone] == 0).all()
