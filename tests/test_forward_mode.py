"""Forward-mode differentiation of the operators that autograd records: refused, where the
tangent would be lost without a word.  Nothing here reaches a GPU."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2506_11209_amd import experts


class OnGpu(torch.Tensor):
    """Stands for a tensor on a GPU."""
    is_cuda = True


def stand_in(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


def dual(*shape):
    return forward_ad.make_dual(stand_in(*shape), torch.ones(*shape))


def test_tangents_are_refused():
    int32 = lambda *shape: stand_in(*shape, dtype=torch.int32)  # noqa: E731
    routes = experts.Routes(int32(5), int32(12), int32(6, 2))
    with forward_ad.dual_level():
        for call in (lambda: experts.choose(dual(6, 8), 2), lambda: experts.gather(dual(6, 8), routes),
                     lambda: experts.combine(dual(12, 8), routes), lambda: experts.combine(stand_in(12, 8), routes, dual(6, 2))):
            with pytest.raises(NotImplementedError):
                call()
            with torch.no_grad(), pytest.raises(NotImplementedError):
                call()


def test_what_has_no_tangent_is_not():
    with forward_ad.dual_level():
        experts._no_forward_mode("choose", stand_in(6, 8), None)
    experts._no_forward_mode("choose", stand_in(6, 8))
