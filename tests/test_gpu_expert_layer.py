"""The layer of experts against the same layer in 64 bits, and its parts together."""
import pytest
import torch

from tests.gpu_helpers import log

expert_layer = pytest.importorskip("paper_2506_11209_amd.expert_layer")

pytestmark = pytest.mark.gpu


def plain(layer, x, ids):
    """y in 64 bits on the CPU with autograd, for the given choices."""
    router, w1, w2 = (p.detach().double().cpu().requires_grad_() for p in (layer.router, layer.w1, layer.w2))
    xd = x.detach().double().cpu().requires_grad_()
    score = (xd @ router.t()).gather(1, ids)
    y = torch.zeros_like(xd)
    weights = score.softmax(1)
    for e in range(w1.shape[0]):
        t, j = (ids == e).nonzero(as_tuple=True)
        rows = torch.nn.functional.silu(xd[t] @ w1[e].t()) @ w2[e].t()
        y = y.index_add(0, t, weights[t, j, None] * rows)
    return y, (xd, router, w1, w2)


def off(a, b):
    b = b.detach()
    return ((a.detach().double().cpu() - b).norm() / b.norm()).item()


@pytest.mark.parametrize("T,columns,hidden,E,k", [(200, 256, 384, 8, 2), (33, 136, 200, 5, 3), (1, 128, 128, 4, 1)])
def test_layer_and_gradients(T, columns, hidden, E, k):
    log("case layer %d tokens, %d of %d experts" % (T, k, E))
    g = torch.Generator(device="cuda").manual_seed(T)
    layer = expert_layer.ExpertLayer(columns, hidden, E, k, generator=g)
    x = torch.randn(T, columns, device="cuda", generator=g).bfloat16().requires_grad_()
    dy = torch.randn(T, columns, device="cuda", generator=g).bfloat16()
    y = layer(x)
    y.backward(dy)
    ids = layer.route(x.detach())[1].cpu()
    want, leaves = plain(layer, x, ids)
    want.backward(dy.double().cpu())
    # A quantised value is off by 2^-4 of itself at most, 2^-4 / sqrt(3) = 3.6 % in the mean square
    # at most; errors of independent factors add in squares.  y has four quantised factors one after
    # the other (7.2 %), the gradients up to seven (9.6 %), silu's slope passes on at most 1.1 of an
    # error; bf16 adds 0.4 %.
    assert off(y, want) <= 0.09
    for got, leaf in ((x.grad, leaves[0]), (layer.router.grad, leaves[1]), (layer.w1.grad, leaves[2]), (layer.w2.grad, leaves[3])):
        assert got.shape == leaf.grad.shape
        if leaf.grad.norm() > 0:
            assert off(got, leaf.grad) <= 0.13
    assert off(layer.serve(x.detach(), layer.serving_weights()), want) <= 0.09


def test_command_runs(capsys):
    log("case layer command")
    capsys.readouterr()
    expert_layer.main(["--tokens", "64", "--decode", "4", "--columns", "256", "--hidden", "256", "--experts", "4", "--steps", "2"])
    lines = capsys.readouterr().out.strip().splitlines()
    assert len(lines) == 2 and "training" in lines[0] and "decoding" in lines[1]
