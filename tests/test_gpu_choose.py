"""The router's choice, its balance loss and its gradient against their definitions in
64 bits.

Tolerances: an exponential is taken of a difference of two values, which rounds, and is
multiplied with log2(e), which rounds again: 2^-23 of the difference, at most 20 for the
logits here, so 2.4e-6 of the exponential; it is itself off by at most 2 steps, and
quotients and sums of up to 1024 of them add 10 steps in a tree and fma chains of up to
64: 4e-6 + 80 * 2^-24 = 9e-6, taken as 1e-5.  Sums over tokens: f32 chains of tokens of a lane, at most 64
here, and a few more adds: within the same.  A result in 16 bits is rounded once."""
import numpy as np
import pytest
import torch

from tests import choose_ref as ref
from tests.gpu_helpers import log

experts = pytest.importorskip("paper_2506_11209_amd.experts")

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
REL = 1e-5


def make(T, E, seed, dtype, masked=0.1, hidden=0.1, ties=False):
    """Logits on the CPU: some tokens masked, some logits of -inf; ties: few values, both zeros."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, E, generator=g) * 2
    if ties:
        x = (x * 1.5).round() * torch.where(torch.rand(T, E, generator=g) < 0.5, -1.0, 1.0)
    x[torch.rand(T, E, generator=g) < hidden] = -torch.inf
    x[torch.rand(T, generator=g) < masked] = -torch.inf
    return x.to(dtype)


def check(x, k, out):
    weights, ids, counts, loss = out
    w, i, c, l, _ = ref.choose(x.double().numpy(), k)
    assert np.array_equal(ids.cpu().numpy(), i)
    assert np.array_equal(counts.cpu().numpy(), c)
    assert np.allclose(weights.cpu().double().numpy(), w, rtol=REL, atol=1e-30)
    assert abs(float(loss) - l) <= REL * l
    assert (weights.dtype, ids.dtype, counts.dtype, loss.dtype, loss.dim()) == (torch.float32, torch.int32, torch.int32, torch.float32, 0)


# around the widths of the rows that lanes hold, and what one workgroup takes
SIZES = [(1, 1, 1), (1, 4, 4), (3, 7, 2), (5, 16, 16), (33, 17, 3), (64, 64, 4), (257, 65, 32), (40, 128, 8), (300, 129, 1), (513, 256, 8),
         (700, 100, 20), (19, 257, 5), (33, 512, 32), (70, 513, 17), (600, 1000, 6), (9, 1024, 32)]


@pytest.mark.parametrize("T,E,k", SIZES)
@pytest.mark.parametrize("name", TYPES)
def test_choose(T, E, k, name):
    log("case choose %d x %d, %d, %s" % (T, E, k, name))
    for ties in (False, True):
        x = make(T, E, T + E + k, TYPES[name], ties=ties)
        check(x, k, experts.choose(x.cuda(), k))


@pytest.mark.parametrize("T,E,k", SIZES)
@pytest.mark.parametrize("name", TYPES)
def test_gradient(T, E, k, name):
    log("case choose gradient %d x %d, %d, %s" % (T, E, k, name))
    x = make(T, E, T * E + k, TYPES[name])
    g = torch.Generator().manual_seed(1)
    dw, dl = torch.randn(T, k, generator=g), torch.tensor(3.0)
    weights, ids, counts, _ = experts.choose(x.cuda(), k)
    for a, b in ((dw, dl), (dw, None), (None, dl), (None, None)):
        got = experts.choose_gradient(a if a is None else a.cuda(), b if b is None else b.cuda(), x.cuda(), weights, ids, counts)
        want = ref.gradient(None if a is None else a.double().numpy(), b, x.double().numpy(), k)
        # terms cancel: errors are relative to their sizes, w |dw| (twice) and the loss's factor times p counts (twice)
        w, i, c, _, p = ref.choose(x.double().numpy(), k)
        size = np.zeros_like(want)
        if a is not None:
            m = w * (np.abs(a.double().numpy()) + (w * np.abs(a.double().numpy())).sum(1, keepdims=True))
            for t in range(T):
                for j in range(k):
                    if i[t, j] >= 0:
                        size[t, i[t, j]] += m[t, j]
        if b is not None and c[E]:
            size += 3.0 * E / (c[:E].sum() * c[E]) * p * (c[:E] + (p * c[:E]).sum(1, keepdims=True))
        step = 0.0 if name == "f32" else torch.finfo(TYPES[name]).eps / 2
        tiny = 0.0 if name != "f16" else 2.0 ** -25  # half a subnormal step
        off = np.abs(got.cpu().double().numpy() - want)
        assert (off <= 2 * REL * size + step * np.abs(want) * (1 + 1e-3) + 2 * REL * step * size + tiny).all()
        assert got.dtype == x.dtype


def test_rows_apart_and_unaligned():
    log("case choose strides")
    big = torch.full((50, 90), 7.0).bfloat16()
    x = make(50, 33, 5, torch.bfloat16)
    big[:, 1:34] = x
    view = big.cuda()[:, 1:34]
    out = experts.choose(view, 3)
    check(x, 3, out)
    dw = torch.randn(50, 3, device="cuda")
    dense = experts.choose_gradient(dw, out[3], x.cuda(), *out[:3])
    into = torch.full((50, 41), 9.0, dtype=torch.bfloat16, device="cuda")
    experts.choose_gradient(dw, out[3], view, *out[:3], out=into[:, 3:36])
    assert torch.equal(into[:, 3:36], dense) and (into[:, :3] == 9).all() and (into[:, 36:] == 9).all()


def test_rows_beyond_32_bits():
    """Rows more than 2^31 elements apart, of logits and of their gradient."""
    log("case choose far apart")
    x = make(4, 40, 8, torch.bfloat16, masked=0.0)
    view = torch.empty(3 * 2**30 + 40, dtype=torch.bfloat16, device="cuda").as_strided((4, 40), (2**30, 1))
    view.copy_(x)
    out = experts.choose(view, 3)
    check(x, 3, out)
    dw = torch.randn(4, 3, device="cuda")
    want = experts.choose_gradient(dw, out[3], x.cuda(), *out[:3])
    assert torch.equal(experts.choose_gradient(dw, out[3], view, *out[:3], out=view), want)


def test_smallest_values():
    """Subnormal logits keep their order, on both sides of the zeros."""
    log("case choose subnormal")
    for dtype, tiny in ((torch.float32, 2.0**-149), (torch.bfloat16, 2.0**-133), (torch.float16, 2.0**-24)):
        x = torch.tensor([[tiny, 3 * tiny, 0.0, -tiny, -0.0, -2 * tiny, 2 * tiny]], dtype=dtype)
        assert experts.choose(x.cuda(), 7)[1].tolist() == [[1, 6, 0, 2, 4, 3, 5]]


def test_nothing_to_choose():
    log("case choose nothing")
    for x in (torch.empty(0, 5), torch.full((3, 5), -torch.inf), torch.full((4000, 5), -torch.inf)):
        weights, ids, counts, loss = experts.choose(x.cuda(), 2)
        assert (weights == 0).all() and (ids == -1).all() and (counts == 0).all() and float(loss) == 0.0
        d = experts.choose_gradient(torch.ones_like(weights), torch.ones((), device="cuda"), x.cuda(), weights, ids, counts)
        assert d.shape == x.shape and (d == 0).all()


def test_infinities_and_nan():
    log("case choose nan")
    nan, inf = float("nan"), float("inf")
    x = torch.tensor([[1.0, nan, 3.0, -inf], [inf, 2.0, inf, 0.0], [0.0, -0.0, 0.0, -0.0], [-inf, -inf, -3e38, 3e38], [nan, nan, -inf, -inf]])
    weights, ids, counts, loss = experts.choose(x.cuda(), 3)
    assert ids.tolist() == [[1, 2, 0], [0, 2, 1], [0, 1, 2], [3, 2, -1], [0, 1, -1]]
    assert counts.tolist() == [4, 4, 4, 1, 5] and loss.isnan()
    w = weights.cpu()
    assert w[0].isnan().all() and w[1].isnan()[:2].all() and w[4, :2].isnan().all() and w[4, 2] == 0
    assert torch.allclose(w[2], torch.tensor(1 / 3)) and w[3].tolist() == [1.0, 0.0, 0.0]
    d = experts.choose_gradient(torch.ones(5, 3, device="cuda"), None, x.cuda(), weights, ids, counts).cpu()
    assert d[2].abs().max() <= 1e-6 and d[3].abs().max() <= 1e-6


def test_same_bits_every_time():
    log("case choose again")
    x = make(9000, 200, 3, torch.float32).cuda()
    first = experts.choose(x, 4)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, experts.choose(x, 4)))


def test_autograd():
    log("case choose autograd")
    x = make(300, 40, 8, torch.float32, hidden=0.0).cuda()
    a = x.clone().requires_grad_()
    weights, ids, counts, loss = experts.choose(a, 3)
    assert not ids.requires_grad and not counts.requires_grad
    dw = torch.randn(300, 3, device="cuda")
    g, = torch.autograd.grad((weights * dw).sum() + 0.5 * loss, a, retain_graph=True)
    assert torch.equal(g, experts.choose_gradient(dw, torch.tensor(0.5, device="cuda"), x, weights, ids, counts))
    g, = torch.autograd.grad(loss, a, retain_graph=True)
    assert torch.equal(g, experts.choose_gradient(None, torch.tensor(1.0, device="cuda"), x, weights, ids, counts))
    g, = torch.autograd.grad(weights.sum(1).expand(2, 300).sum(), a, retain_graph=True)  # softmax sums to 1
    assert g.abs().max() <= 1e-6
    with pytest.raises(RuntimeError):
        g, = torch.autograd.grad(loss, a, create_graph=True)
        g.sum().backward()
    with torch.no_grad():
        assert not experts.choose(a, 3)[0].requires_grad


def test_gradient_against_differences():
    """Along random directions, in which the choice does not change: (f(x + h d) - f(x - h d)) / 2 h
    with f in 64 bits by the definition, within h^2 of third derivatives (below 40 for these sizes)
    and the gradient's own tolerance."""
    log("case choose differences")
    x = make(40, 12, 4, torch.float32, masked=0.0, hidden=0.1)
    k, g = 3, np.random.default_rng(0)
    dw = g.standard_normal((40, k)).astype(np.float32)
    weights, ids, counts, _ = experts.choose(x.cuda(), k)
    grad = experts.choose_gradient(torch.from_numpy(dw).cuda(), torch.tensor(2.0, device="cuda"), x.cuda(), weights, ids, counts)
    grad, base = grad.cpu().double().numpy(), x.double().numpy()

    def f(v):
        w, i, _, l, _ = ref.choose(v, k)
        assert np.array_equal(i, ids.cpu().numpy())
        return (w * dw).sum() + 2.0 * l

    h = 1e-4
    for _ in range(5):
        d = np.where(np.isinf(base), 0.0, g.standard_normal(base.shape))
        d /= np.linalg.norm(d)
        with np.errstate(invalid="ignore"):
            slope = (f(base + h * d) - f(base - h * d)) / (2 * h)
        assert abs(slope - (grad * d).sum()) <= 40 * h * h + 1e-9 / h * 1e-3 + 4e-5 * np.abs(grad).max()


def test_captured_and_replayed():
    log("case choose graph")
    x = [make(5000, 64, s, torch.bfloat16).cuda() for s in range(3)]
    at = x[0].clone()
    dw, dl = torch.randn(5000, 4, device="cuda"), torch.tensor(0.3, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = experts.choose(at, 4)
        experts.choose_gradient(dw, dl, at, *out[:3])
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = experts.choose(at, 4)
        d = experts.choose_gradient(dw, dl, at, *out[:3])
    for s in (1, 2, 0, 1):
        at.copy_(x[s])
        graph.replay()
        torch.cuda.synchronize()
        want = experts.choose(x[s], 4)
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert torch.equal(d, experts.choose_gradient(dw, dl, x[s], *want[:3]))


def test_on_another_stream():
    log("case choose stream")
    x = make(3000, 64, 2, torch.float32).cuda()
    want = experts.choose(x, 2)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = experts.choose(x, 2, stream=side)
    dw = torch.ones(3000, 2, device="cuda")
    torch.cuda.synchronize()
    d = experts.choose_gradient(dw, None, x, *out[:3], stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert torch.equal(d, experts.choose_gradient(dw, None, x, *want[:3]))


def test_two_calls_at_once():
    log("case choose two streams")
    x = [make(20000, 200, s, torch.bfloat16).cuda() for s in range(2)]
    want = [experts.choose(v, 4) for v in x]
    streams = [torch.cuda.Stream() for _ in x]
    torch.cuda.synchronize()
    got = [(i, experts.choose(x[i], 4, stream=streams[i])) for _ in range(4) for i in range(2)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i, out in got for a, b in zip(out, want[i]))


def test_an_id_twice_beside_others():
    """A token with an id twice leaves the others of its wave as they are."""
    log("case choose twice")
    x = make(8, 64, 4, torch.float32, masked=0.0, hidden=0.0).cuda()
    out = experts.choose(x, 4)
    dw = torch.randn(8, 4, device="cuda")
    want = experts.choose_gradient(dw, out[3], x, *out[:3])
    ids = out[1].clone()
    ids[2, 3] = ids[2, 0]
    got = experts.choose_gradient(dw, out[3], x, out[0], ids, out[2])
    others = [t for t in range(8) if t != 2]
    assert torch.equal(got[others], want[others])
    w, g = out[0][2].double(), dw[2].double()
    asked = w * (g - (w * g).sum())
    change = torch.zeros(64, dtype=torch.float64, device="cuda")
    change[ids[2, 0].long()] += asked[3]
    change[out[1][2, 3].long()] -= asked[3]
    # four values rounded at most eight times each, of at most twice the largest product
    assert ((got[2] - want[2]).double() - change).abs().max() <= 64 * 2.0**-24 * float((w.max() * g.abs().max() * 2 + want[2].abs().max()))


def test_refusals():
    log("case choose refusals")
    x = torch.zeros(6, 8, device="cuda")
    for call in (lambda: experts.choose(x, 0), lambda: experts.choose(x, 9), lambda: experts.choose(x, -1),
                 lambda: experts.choose(torch.zeros(6, 100, device="cuda"), 33), lambda: experts.choose(torch.zeros(6, 1025, device="cuda"), 2),
                 lambda: experts.choose(x.cpu(), 2), lambda: experts.choose(x.double(), 2), lambda: experts.choose(x.t(), 2),
                 lambda: experts.choose(x[0], 1), lambda: experts.choose(torch.zeros(1, 8, device="cuda").expand(6, 8), 2)):
        with pytest.raises(ValueError):
            call()
    w, i, c, l = experts.choose(x, 2)
    dw = torch.ones_like(w)
    for args in ((dw[:5], l, x, w, i, c), (dw, l, x, w[:5], i, c), (dw, l, x, w, i[:5], c), (dw, l, x, w, i.long(), c), (dw, l, x, w, i, c[:8]),
                 (dw, torch.zeros(2, device="cuda"), x, w, i, c), (dw, l.double(), x, w, i, c), (dw.t().contiguous().t(), l, x, w, i, c),
                 (dw.cpu(), l, x, w, i, c), (dw, l, x, None, i, c)):
        with pytest.raises(ValueError):
            experts.choose_gradient(*args)
    with pytest.raises(ValueError):
        experts.choose_gradient(dw, l, x, w, i, c, out=torch.zeros(6, 7, device="cuda"))
    # ids out of range, as a caller's own could be, count as none
    bad = i.clone()
    bad[0, 0], bad[1, 1] = 8, -5
    d = experts.choose_gradient(dw, None, x, w, bad, c)
    assert d.isfinite().all()
    # the same id twice: both its parts arrive
    twice = torch.tensor([[3, 3]], dtype=torch.int32, device="cuda")
    w, dw = torch.tensor([[0.25, 0.5]], device="cuda"), torch.tensor([[1.0, 2.0]], device="cuda")
    d = experts.choose_gradient(dw, None, x[:1], w, twice, c)
    assert d.tolist() == [[0, 0, 0, 0.25 * (1 - 1.25) + 0.5 * (2 - 1.25), 0, 0, 0, 0]]
