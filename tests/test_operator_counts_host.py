"""Counts that do not fit the library's 32 bits, or are negative, are refused by the
Python calls that take them and not cut (CPU only)."""
import pytest
import torch

from paper_2506_11209_amd import experts, fp8

TOO_MANY = ((1 << 32) + 4, 1 << 31, -(1 << 32) + 4, (1 << 64) + 4, -1)


class Ids(torch.Tensor):
    """Stands for tokens x k on a GPU."""
    is_cuda = True


@pytest.mark.parametrize("count", TOO_MANY)
def test_experts(count):
    ids = torch.zeros(6, 2, dtype=torch.int32).as_subclass(Ids)
    with pytest.raises(ValueError):
        experts.sort(ids, count)


@pytest.mark.parametrize("count", TOO_MANY)
def test_groups(count):
    with pytest.raises(ValueError):
        fp8.padded_rows(100, count)
    with pytest.raises((ValueError, fp8._w.WsGemmError)):
        fp8.plan(10, 10, 10, groups=count)


@pytest.mark.parametrize("rows", (-1, (1 << 30) + 1, (1 << 64) + 4))
def test_rows(rows):
    with pytest.raises(ValueError):
        fp8.padded_rows(rows, 2)
    for sizes in ((rows, 10, 10), (10, rows, 10), (10, 10, rows)):
        with pytest.raises((ValueError, fp8._w.WsGemmError)):
            fp8.plan(*sizes)
