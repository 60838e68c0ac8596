"""What OrthogonalMomentum refuses, before anything has changed.  Nothing here reaches a GPU."""
import pytest
import torch

from paper_2506_11209_amd import orthogonal


def parameter(*shape, dtype=torch.float32, device="meta"):
    return torch.nn.Parameter(torch.empty(*shape, dtype=dtype, device=device))


@pytest.mark.parametrize("shape", [(65537, 8), (8, 65537), (1 << 17, 5, 5), (64, 65536, 65536), (1 << 32, 1)])
def test_sizes_that_no_launch_holds(shape):
    with pytest.raises(ValueError):
        orthogonal.OrthogonalMomentum([parameter(*shape)])
    optimizer = orthogonal.OrthogonalMomentum([parameter(4, 8)])
    with pytest.raises(ValueError):
        optimizer.add_param_group({"params": [parameter(5, 5), parameter(*shape)]})
    assert len(optimizer.param_groups) == 1


@pytest.mark.parametrize("bad", [dict(steps=0), dict(steps=101), dict(steps=2.5), dict(steps=5.0), dict(momentum=1.0), dict(momentum=-0.1), dict(lr=-1e-3),
                                 dict(weight_decay=-1.0), dict(lr=float("nan"))])
def test_options_of_a_group(bad):
    with pytest.raises(ValueError):
        orthogonal.OrthogonalMomentum([{"params": [parameter(4, 8)], **bad}])
    with pytest.raises(ValueError):
        orthogonal.OrthogonalMomentum([parameter(4, 8)], **bad)
    optimizer = orthogonal.OrthogonalMomentum([parameter(4, 8)])
    with pytest.raises(ValueError):
        optimizer.add_param_group({"params": [parameter(4, 8)], **bad})
    assert len(optimizer.param_groups) == 1
    optimizer.param_groups[0].update(bad)  # as a schedule or a loaded state may
    with pytest.raises(ValueError):
        optimizer.step()


def test_gradients_before_any_change():
    """One gradient that no kernel takes: no parameter and no momentum has changed."""
    for bad in (torch.zeros(4, 8).to_sparse(), torch.zeros(4, 8), torch.zeros(4, 8, dtype=torch.float64)):
        p, q = parameter(4, 8, device="cpu"), parameter(4, 8, dtype=bad.dtype, device="cpu")
        with torch.no_grad():
            p.fill_(1.0)
        optimizer = orthogonal.OrthogonalMomentum([p, q], weight_decay=0.5)
        p.grad, q.grad = torch.ones(4, 8).as_subclass(OnGpu), bad
        with pytest.raises(ValueError):
            optimizer.step()
        assert (p == 1).all() and not optimizer.state


class OnGpu(torch.Tensor):
    """Stands for a tensor on a GPU."""
    is_cuda = True
