"""A call that is refused leaves the caller's current device and stream as they
were (CPU only: torch's contexts are recorded)."""
import pytest
import torch

from paper_2506_11209_amd import fp8


class Stream:
    def __init__(self, device):
        self.device = device


class Tensor:
    """Stands for a tensor that a stream cannot be recorded on, as one on the CPU."""
    is_cuda = False
    device = torch.device("cpu")

    def record_stream(self, stream):
        raise NotImplementedError("record_stream on the CPU")


@pytest.fixture
def entered(monkeypatch):
    """What has been entered and not left."""
    now = []

    def context(what):
        class Context:
            def __init__(self, value):
                self.entry = (what, value)

            def __enter__(self):
                now.append(self.entry)

            def __exit__(self, *exc):
                now.remove(self.entry)

        return Context

    monkeypatch.setattr(torch.cuda, "device", context("device"))
    monkeypatch.setattr(torch.cuda, "stream", context("stream"))
    return now


DEVICE = torch.device("cuda", 0)


def test_a_stream_of_another_device(entered):
    with pytest.raises(ValueError):
        with fp8._Call(DEVICE, Stream(torch.device("cuda", 1)), []):
            pass
    assert entered == []


def test_an_operand_that_is_not_on_the_device(entered):
    """It is left to the call's own checks, which raise ValueError."""
    stream = Stream(DEVICE)
    for operand in (Tensor(), "no tensor", 3):
        with fp8._Call(DEVICE, stream, [None, operand]):
            assert entered == [("device", DEVICE), ("stream", stream)]
        assert entered == []


def test_an_error_while_entering(entered):
    class Broken(torch.Tensor):
        is_cuda = True
        device = DEVICE

        def record_stream(self, stream):
            raise RuntimeError("no record")

    with pytest.raises(RuntimeError, match="no record"):
        with fp8._Call(DEVICE, Stream(DEVICE), [Broken()]):
            pass
    assert entered == []


def test_without_a_stream(entered):
    with fp8._Call(DEVICE, None, [Tensor()]):
        assert entered == [("device", DEVICE)]
    assert entered == []
