"""Orthogonalised updates against the iteration in 64 bits.

Tolerances.  Binary16 rounds by u = 2^-11 of a value.  A step from X, with |.| the
Frobenius and ||.|| the spectral norm: the operand of A = X X^T is off by u |X|, so A by
2 u |X| ||X||, and off the diagonal by u |S| more where it is stored; T = b A + c A^2 by
(|b| + 2 |c| ||A||) times that, and by u |T| (off the diagonal) where it is stored; the new
X by that times ||X||, and by ||T|| (off the diagonal) u |X| for its operand.  Sums in
binary32 and the rest of X, which is kept, add less than a tenth to these.  What a step
leaves, the later ones take along at the most by L, the larger of the largest |p'(s)| and
p(s) / s over the singular values s that there are (with a twentieth around them), p(s) =
a s + b s^3 + c s^5.  The result rounds to bf16 by 2^-8 of a value at the most.

Where S and T have nothing off their diagonals, or nothing rounds, the tests compare
value by value."""
import math

import numpy as np
import pytest
import torch

from tests.gpu_helpers import log

orthogonal = pytest.importorskip("paper_2506_11209_amd.orthogonal")

pytestmark = pytest.mark.gpu

A, B, CUBE = 3.4445, -4.7750, 2.0315
U, OUT = 2.0 ** -11, 2.0 ** -8
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def iterate(G, steps):
    """(result, bound on its error before the last rounding, Frobenius) for one matrix in 64 bits."""
    X = G.double().cpu().numpy()
    X = X / np.linalg.norm(X)
    tall = X.shape[0] > X.shape[1]
    X = X.T if tall else X
    error = 0.0
    for _ in range(steps):
        s = np.linalg.svd(X, compute_uv=False)
        M = X @ X.T
        T = B * M + CUBE * M @ M
        off_m, off_t = M - np.diag(np.diag(M)), T - np.diag(np.diag(T))
        top, fro = s[0], np.linalg.norm(X)
        d_m = 2 * U * fro * top + U * np.linalg.norm(off_m)
        d_t = (abs(B) + 2 * CUBE * top ** 2) * d_m + U * np.linalg.norm(off_t)
        local = 1.1 * (d_t * top + np.linalg.norm(off_t, 2) * U * fro)
        g = np.linspace(0.95 * s[-1], 1.05 * s[0], 2000)
        L = max(np.abs(A + 3 * B * g ** 2 + 5 * CUBE * g ** 4).max(), np.abs(A + B * g ** 2 + CUBE * g ** 4).max())
        error = L * error + local
        X = A * X + T @ X
    return (X.T if tall else X), error


def check(got, G, steps=5):
    want, error = iterate(G, steps)
    got = got.double().cpu().numpy()
    bound = error * (1 + OUT) + OUT * np.linalg.norm(want)
    assert np.linalg.norm(got - want) <= bound, (np.linalg.norm(got - want), bound)
    return np.linalg.norm(got - want) / np.linalg.norm(want)


def spread(shape, seed, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.where(torch.rand(shape[-1], generator=g) < 0.02, 5.0, 1.0)
    return (x * 1e-2).to(dtype)


SHAPES = [(1, 1), (1, 5), (7, 1), (2, 64), (17, 33), (64, 64), (65, 130), (200, 63), (63, 200), (128, 128), (129, 257), (300, 120), (16, 2048),
          (2000, 24), (400, 500)]


@pytest.mark.parametrize("R,C", SHAPES)
@pytest.mark.parametrize("name", TYPES)
def test_against_64_bits(R, C, name):
    log("case orthogonalize %d x %d %s" % (R, C, name))
    G = spread((R, C), R * C, TYPES[name])
    for steps in (1, 2, 5):
        off = check(orthogonal.orthogonalize(G.cuda(), steps), G, steps)
        log("  %d steps: %.2e" % (steps, off))


@pytest.mark.parametrize("R,C", [(600, 1100), (1100, 600), (513, 513), (257, 4100)])
def test_several_tiles(R, C):
    log("case orthogonalize tiles %d x %d" % (R, C))
    G = spread((R, C), 1)
    check(orthogonal.orthogonalize(G.cuda()), G)


def scalar(x, steps):
    for _ in range(steps):
        x = A * x + B * x ** 3 + CUBE * x ** 5
    return x


@pytest.mark.parametrize("R,C", [(1, 1), (5, 3), (64, 64), (70, 200), (300, 129), (520, 700), (1000, 260), (2100, 1300)])
def test_signed_permutations(R, C):
    """One entry in each row and column of the shorter side: S and T are diagonal, and every entry goes its own way."""
    log("case orthogonalize permutation %d x %d" % (R, C))
    g = torch.Generator().manual_seed(R)
    n = min(R, C)
    rows, cols = torch.randperm(R, generator=g)[:n], torch.randperm(C, generator=g)[:n]
    size = torch.randint(1, 4, (n,), generator=g).double() * torch.where(torch.rand(n, generator=g) < 0.5, -1.0, 1.0)
    G = torch.zeros(R, C)
    G[rows, cols] = (size * 0.125).float()
    got = orthogonal.orthogonalize(G.cuda()).cpu().double()
    want = torch.zeros(R, C, dtype=torch.float64)
    want[rows, cols] = scalar(size / size.norm(), 5)
    # the operand of A alone is rounded: u of a value a step, squared and times |b| s^2 .., all of it less than u each
    slope = 3.5 ** 5
    assert ((got - want).abs() <= OUT * want.abs() + 2e-4 * want.abs() + slope * 2 * U * (size.abs().max() / size.norm()) ** 2 * (want != 0)).all()
    assert (got[want == 0] == 0).all()


@pytest.mark.parametrize("R,C", [(4, 4), (64, 64), (16, 64), (256, 64), (128, 128), (128, 512), (1024, 256), (256, 256), (512, 512)])
def test_one_step_of_signs(R, C):
    """Entries of +-1 whose norm is a power of two: X, A and A^2 are exact, T rounds once off its diagonal."""
    log("case orthogonalize signs %d x %d" % (R, C))
    g = torch.Generator().manual_seed(R + C)
    G = torch.where(torch.rand(R, C, generator=g) < 0.5, -1.0, 1.0)
    X = G.double().numpy() / math.sqrt(R * C)
    X = X.T if R > C else X
    M = X @ X.T
    T = B * M + CUBE * M @ M
    want = A * X + T @ X
    off = np.abs(T - np.diag(np.diag(T)))
    bound = (OUT * np.abs(want) + U * off @ np.abs(X)) * (1 + 1e-3) + 1e-5 * np.abs(X).max()
    got = orthogonal.orthogonalize(G.cuda(), 1).double().cpu().numpy()
    got = got.T if R > C else got
    assert (np.abs(got - want) <= bound).all()


def test_powers_of_two_change_nothing():
    log("case orthogonalize scale")
    G = spread((90, 150), 2)
    want = orthogonal.orthogonalize(G.cuda())
    for e in (-90, 40, 110):
        assert torch.equal(orthogonal.orthogonalize((G * 2.0 ** e).cuda()), want)
    tiny = torch.zeros(3, 70)
    tiny[1, 5] = 1e-45  # the smallest there is
    assert abs(float(orthogonal.orthogonalize(tiny.cuda())[1, 5]) - scalar(1.0, 5)) <= OUT


def test_batch_and_strides():
    log("case orthogonalize batch")
    big = spread((5, 70, 210), 3).cuda()
    G = big[1:4, 2:67, 3:203]
    got = orthogonal.orthogonalize(G)
    for i in range(3):
        assert torch.equal(got[i], orthogonal.orthogonalize(G[i].contiguous()))
    into = torch.full((3, 70, 210), 7.0, dtype=torch.bfloat16, device="cuda")
    out = into[:, 1:66, 5:205]
    assert orthogonal.orthogonalize(G, out=out) is out
    assert torch.equal(out, got)
    out.fill_(7.0)
    assert (into == 7).all()
    # a tall batch, whose results lie the other way round
    T = G.transpose(1, 2).contiguous()
    tall, into = orthogonal.orthogonalize(T), torch.full((3, 203, 71), 7.0, dtype=torch.bfloat16, device="cuda")
    assert torch.equal(tall, got.transpose(1, 2))
    orthogonal.orthogonalize(T, out=into[:, 3:, 6:])
    assert torch.equal(into[:, 3:, 6:], tall) and (into[:, :3] == 7).all() and (into[..., :6] == 7).all()


def test_many_matrices():
    """More tiles than the card has room for at once, of both tile sizes."""
    log("case orthogonalize many")
    G = spread((40, 600, 700), 4)
    got = orthogonal.orthogonalize(G.cuda())
    assert torch.equal(got[39], orthogonal.orthogonalize(G[39].cuda()))
    check(got[17], G[17])
    G = spread((300, 20, 30), 5)
    got = orthogonal.orthogonalize(G.cuda())
    for i in (0, 299):
        check(got[i], G[i])


def test_zeros_infinities_and_nan():
    log("case orthogonalize nan")
    G = spread((6, 80, 100), 6)
    G[1] = 0.0
    G[2, 3, 4], G[3, 79, 99], G[4, 0, 0] = float("nan"), float("inf"), float("-inf")
    G[5, 40:] = 0.0  # rows without a gradient
    got = orthogonal.orthogonalize(G.cuda())
    assert (got[1] == 0).all() and got[2:5].isnan().all() and (got[5, 40:] == 0).all()
    assert torch.equal(got[0], orthogonal.orthogonalize(G[0].cuda()))
    check(got[5, :40], G[5, :40])


def test_nothing():
    log("case orthogonalize nothing")
    for shape in ((0, 5), (5, 0), (0, 4, 4), (3, 0, 7)):
        got = orthogonal.orthogonalize(torch.empty(shape, device="cuda"))
        assert got.shape == shape and got.dtype == torch.bfloat16


def test_captured_and_on_a_stream():
    log("case orthogonalize graph")
    G = [spread((4, 130, 260), s).cuda() for s in range(3)]
    want = [orthogonal.orthogonalize(g) for g in G]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = orthogonal.orthogonalize(G[1], stream=side)
    side.synchronize()
    assert torch.equal(got, want[1])
    at, graph = G[0].clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = orthogonal.orthogonalize(at)
    for s in (1, 2, 0, 2):
        at.copy_(G[s])
        graph.replay()
        eager = orthogonal.orthogonalize(G[s])
        torch.cuda.synchronize()
        assert torch.equal(out, want[s]) and torch.equal(eager, want[s])


def test_two_calls_at_once():
    log("case orthogonalize two streams")
    G = [spread((900, 1200), s).cuda() for s in range(2)]
    want = [orthogonal.orthogonalize(g) for g in G]
    streams = [torch.cuda.Stream() for _ in G]
    torch.cuda.synchronize()
    got = [orthogonal.orthogonalize(g, stream=s) for g, s in zip(G, streams) for _ in range(2)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i // 2]) for i, o in enumerate(got))


def test_optimizer():
    log("case orthogonal momentum")
    g = torch.Generator().manual_seed(0)
    w = [torch.nn.Parameter(torch.randn(s, generator=g).cuda()) for s in ((3, 60, 40), (20, 70))]
    start, grads = [p.detach().clone() for p in w], [[torch.randn(p.shape, generator=g).cuda() for p in w] for _ in range(2)]
    opt = orthogonal.OrthogonalMomentum(w, lr=0.1, momentum=0.9, weight_decay=0.01)
    for step in range(2):
        for p, d in zip(w, grads[step]):
            p.grad = d.clone()
        opt.step()
    for p, s, a, b in zip(w, start, *grads):
        factor = 0.1 * max(1.0, p.shape[-2] / p.shape[-1]) ** 0.5
        for u in (a + 0.9 * a, b + 0.9 * (0.9 * a + b)):
            s = s * (1 - 0.1 * 0.01) - factor * orthogonal.orthogonalize(u).float()
        assert (p - s).abs().max() <= 1e-2 * factor  # u rounds otherwise here: its update by far less than this
    for bad in (dict(lr=-1.0), dict(momentum=1.0), dict(steps=0)):
        with pytest.raises(ValueError):
            orthogonal.OrthogonalMomentum(w, **bad)
    with pytest.raises(ValueError):
        orthogonal.OrthogonalMomentum([torch.nn.Parameter(torch.zeros(3, device="cuda"))])


def test_optimizer_keeps_momentum_in_32_bits():
    log("case orthogonal momentum of bf16")
    g = torch.Generator().manual_seed(1)
    w = torch.randn(30, 50, generator=g).bfloat16()
    grads = [torch.randn(30, 50, generator=g).bfloat16().cuda() for _ in range(3)]

    def run(steps, opt):
        for d in steps:
            opt.param_groups[0]["params"][0].grad = d.clone()
            opt.step()

    one = orthogonal.OrthogonalMomentum([torch.nn.Parameter(w.cuda())], lr=0.1, momentum=0.9)
    run(grads[:2], one)
    p = one.param_groups[0]["params"][0]
    b = one.state[p]["momentum"]
    assert b.dtype == torch.float32 and torch.equal(b, torch.zeros_like(b).add_(grads[0]).mul_(0.9).add_(grads[1]))
    other = orthogonal.OrthogonalMomentum([torch.nn.Parameter(p.detach().clone())], lr=0.5)
    other.load_state_dict(one.state_dict())
    run(grads[2:], one)
    run(grads[2:], other)
    q = other.param_groups[0]["params"][0]
    assert torch.equal(p, q) and torch.equal(one.state[p]["momentum"], other.state[q]["momentum"])


def test_refusals():
    log("case orthogonalize refusals")
    G = torch.zeros(6, 8, device="cuda")
    for call in (lambda: orthogonal.orthogonalize(G, 0), lambda: orthogonal.orthogonalize(G, 101), lambda: orthogonal.orthogonalize(G.cpu()),
                 lambda: orthogonal.orthogonalize(G.double()), lambda: orthogonal.orthogonalize(G.t()), lambda: orthogonal.orthogonalize(G[0]),
                 lambda: orthogonal.orthogonalize(G, out=torch.zeros(6, 8, device="cuda")),
                 lambda: orthogonal.orthogonalize(G, out=torch.zeros(6, 7, dtype=torch.bfloat16, device="cuda")),
                 lambda: orthogonal.orthogonalize(G, out=torch.zeros(6, 8, dtype=torch.bfloat16)),
                 lambda: orthogonal.orthogonalize(torch.zeros(1, 65537, device="cuda")),
                 lambda: orthogonal.orthogonalize(torch.zeros(1, 8, device="cuda").expand(6, 8))):
        with pytest.raises(ValueError):
            call()
