"""Gradients through gather, combine and the layer of experts by torch's autograd:
none gets lost, none is computed that nobody asked for, and what is kept for the
way back goes where torch's hooks for saved tensors send it."""
import numpy as np
import pytest
import torch

from tests import fp8_ref as ref
from tests.gpu_helpers import log
from tests.test_gpu_experts import make_ids

fp8 = pytest.importorskip("paper_2506_11209_amd.fp8")
experts = pytest.importorskip("paper_2506_11209_amd.experts")
expert_layer = pytest.importorskip("paper_2506_11209_amd.expert_layer")

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
T, k, E, C = 40, 3, 6, 72


def routes(seed=1):
    ids = make_ids(T, k, E, seed, 0.2)
    ids[3] = -1
    r = experts.sort(ids.cuda(), E)
    return r, r.place.cpu().long()


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_gather(dtype):
    log("case gradient of gather %s" % dtype)
    typ, (r, place) = TYPES[dtype], routes()
    g = torch.Generator().manual_seed(2)
    x, dxs = torch.randn(T, C, generator=g).to(typ), torch.randn(T * k, C, generator=g).to(typ)
    xd = x.cuda().requires_grad_()
    xs = experts.gather(xd, r)
    assert torch.equal(xs.detach(), experts.gather(x.cuda(), r))
    xs.backward(dxs.cuda())
    want, size = np.zeros((T, C)), np.zeros((T, C))
    for t in range(T):
        for j in range(k):
            if place[t, j] >= 0:
                want[t] += ref.f64(dxs)[place[t, j]]
                size[t] += np.abs(ref.f64(dxs)[place[t, j]])
    # k additions in binary32, one rounding (f16 subnormals: 2^-25)
    ref.assert_within(ref.f64(xd.grad), want, (k + 1) * 2.0 ** -24 * size + 1.01 * ref.HALF_ULP[typ] * np.abs(want) + 2.0 ** -25 * (typ == torch.float16))


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_combine(dtype):
    log("case gradient of combine %s" % dtype)
    typ, (r, _) = TYPES[dtype], routes()
    g = torch.Generator().manual_seed(3)
    h, w, dy = (torch.randn(*s, generator=g).cuda() for s in ((T * k, C), (T, k), (T, C)))
    h, dy = h.to(typ), dy.to(typ)
    want_h, want_w = experts.combine_gradient(dy, h, r, w)  # compared with the formula by its own test
    plain_h, _ = experts.combine_gradient(dy, None, r)
    for of_h, of_w in ((True, True), (True, False), (False, True)):
        hd, wd = h.clone().requires_grad_(of_h), w.clone().requires_grad_(of_w)
        y = experts.combine(hd, r, wd)
        assert torch.equal(y.detach(), experts.combine(h, r, w))
        y.backward(dy)
        assert torch.equal(hd.grad, want_h) if of_h else hd.grad is None
        assert torch.equal(wd.grad, want_w) if of_w else wd.grad is None
    hd = h.clone().requires_grad_()
    experts.combine(hd, r).backward(dy)
    assert torch.equal(hd.grad, plain_h)


def test_gradients_that_are_not_dense():
    """A sum's gradient is one value expanded; a transpose's has its columns apart."""
    log("case gradients not dense")
    r, place = routes()
    x = torch.randn(T, C, device="cuda", requires_grad=True)
    xs = experts.gather(x, r)
    xs.sum().backward()
    assert torch.equal(x.grad.cpu(), (place >= 0).sum(1, keepdim=True).float().expand(T, C))
    h, d = torch.randn(T * k, C, device="cuda", requires_grad=True), torch.randn(C, T, device="cuda")
    (experts.combine(h, r).t() * d).sum().backward()
    assert torch.equal(h.grad, experts.combine_gradient(d.t().contiguous(), None, r)[0])


def test_gradients_against_differences():
    """Through both calls and what lies between them, along random directions."""
    log("case autograd differences")
    r, _ = routes()
    g = torch.Generator().manual_seed(4)
    x, w, dy = (torch.randn(*s, generator=g).cuda() for s in ((T, C), (T, k), (T, C)))
    loss = lambda a, b: (dy.double() * experts.combine(experts.gather(a, r).square(), r, b).double()).sum()  # noqa: E731
    xd, wd = x.clone().requires_grad_(), w.clone().requires_grad_()
    loss(xd, wd).backward()
    u, v, s = torch.randn(T, C, generator=g).cuda(), torch.randn(T, k, generator=g).cuda(), 2.0 ** -4
    # The loss is quadratic in x and linear in w, so central differences are exact but for roundings:
    # each of T C outputs is off by (k + 4) 2^-24 of its terms (about k * 3), with random signs
    # sqrt(T C) * 7 * 2^-24 * 9 = 2e-4, over 2 s = 1/8
    for got, diff in (((xd.grad.double() * u.double()).sum(), loss(x + s * u, w) - loss(x - s * u, w)),
                      ((wd.grad.double() * v.double()).sum(), loss(x, w + s * v) - loss(x, w - s * v))):
        assert abs(diff.item() / (2 * s) - got.item()) <= 2e-2 < 0.01 * abs(got.item())


def test_results_in_the_callers_memory_are_not_recorded():
    log("case out and gradients")
    r, _ = routes()
    x, h = torch.randn(T, C, device="cuda", requires_grad=True), torch.randn(T * k, C, device="cuda")
    w = torch.rand(T, k, device="cuda", requires_grad=True)
    for call in (lambda: experts.gather(x, r, out=torch.empty(T * k, C, device="cuda")),
                 lambda: experts.combine(h, r, w, out=torch.empty(T, C, device="cuda"))):
        with pytest.raises(ValueError):
            call()
        with torch.no_grad():
            assert not call().requires_grad
    assert not experts.gather(x.detach(), r).requires_grad


def test_on_another_stream():
    log("case gradients on a stream")
    r, _ = routes()
    x, dy = torch.randn(T, C, device="cuda", requires_grad=True), torch.randn(T, C, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = experts.combine(experts.gather(x, r, stream=side), r, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    y.backward(dy)
    torch.cuda.synchronize()
    assert torch.equal(x.grad, experts.combine(experts.combine_gradient(dy, None, r)[0], r))


def test_second_derivatives_are_refused():
    """They are not computed, so asking for them raises."""
    log("case second derivatives")
    r, _ = routes()
    x, w = torch.randn(T, C, device="cuda", requires_grad=True), torch.rand(T, k, device="cuda", requires_grad=True)
    for y in (experts.gather(x, r).square(), experts.combine(experts.gather(x, r), r, w).square()):
        d, = torch.autograd.grad(y.sum(), x, create_graph=True)
        with pytest.raises(RuntimeError):
            d.square().sum().backward()


def make_layer(seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    layer = expert_layer.ExpertLayer(136, 200, 5, 3, generator=g)
    x = torch.randn(33, 136, device="cuda", generator=g).bfloat16()
    return layer, x, torch.randn(33, 136, device="cuda", generator=g).bfloat16()


def grads(layer, x, dy):
    layer.zero_grad()
    xd = x.clone().requires_grad_()
    layer(xd).backward(dy)
    return {"x": xd.grad, "router": layer.router.grad, "w1": layer.w1.grad, "w2": layer.w2.grad}


def test_layer_refuses_second_derivatives():
    log("case second derivatives of the layer")
    layer, x, _ = make_layer()
    x.requires_grad_()
    d, = torch.autograd.grad(layer(x).float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        d.float().square().sum().backward()


def test_layer_computes_what_is_asked_for(monkeypatch):
    log("case layer frozen weights")
    layer, x, dy = make_layer()
    want = grads(layer, x, dy)
    calls = []
    for name in ("grouped_gradient", "grouped_product", "quantize_both"):
        f = getattr(fp8, name)
        monkeypatch.setattr(fp8, name, lambda *a, _f=f, _n=name, **kw: (calls.append(_n), _f(*a, **kw))[1])

    def count():
        c = [calls.count(n) for n in ("grouped_gradient", "grouped_product", "quantize_both")]
        calls.clear()
        return c

    grads(layer, x, dy)
    assert count() == [2, 4, 4]  # weight gradients; products forward and back; operands in both forms
    for frozen in (("w1",), ("w2",), ("w1", "w2")):
        for name in ("w1", "w2"):
            getattr(layer, name).requires_grad_(name not in frozen)
        got = grads(layer, x, dy)
        assert count()[0] == 2 - len(frozen)
        for name, value in got.items():
            assert value is None if name in frozen else torch.equal(value, want[name])
    layer.zero_grad()
    for name in ("w1", "w2"):
        getattr(layer, name).requires_grad_(False)
    layer(x).backward(dy)  # only the router learns
    assert count() == [0, 2, 0] and torch.equal(layer.router.grad, want["router"])
    assert torch.equal(layer(x).detach(), layer.serve(x, layer.serving_weights()))


def test_layer_keeps_its_operands_as_saved_tensors():
    log("case layer saved tensors")
    layer, x, dy = make_layer()
    want, kept = grads(layer, x, dy), []

    def pack(t):
        kept.append(t.numel() * t.element_size())
        return t.cpu()

    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t.cuda()):
        got = grads(layer, x, dy)
    for name in want:
        assert torch.equal(got[name], want[name])
    # the transposed weights' codes, of 136 and of 200 columns padded to 16, and the rows' of 99 choices
    weights = 5 * (136 * 208 + 200 * 144)
    assert sum(kept) >= weights + 99 * (136 + 200)
    y = layer(x.clone().requires_grad_())
    y.backward(dy)
    with pytest.raises(RuntimeError):  # they are gone
        y.backward(dy)


def test_layer_of_no_tokens():
    log("case layer of nothing")
    layer, x, dy = make_layer()
    got = grads(layer, x[:0], dy[:0])
    assert got["x"].shape == (0, 136)
    for name in ("router", "w1", "w2"):
        assert torch.equal(got[name], torch.zeros_like(getattr(layer, name)))
