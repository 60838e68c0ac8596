"""Refused calls on a stream of the caller's: ValueError, and the current stream
stays the caller's."""
import pytest
import torch

from tests.gpu_helpers import log

fp8 = pytest.importorskip("paper_2506_11209_amd.fp8")
experts = pytest.importorskip("paper_2506_11209_amd.experts")

pytestmark = pytest.mark.gpu


def test_refused_calls_keep_the_current_stream():
    log("case refused on a stream")
    side, before = torch.cuda.Stream(), torch.cuda.current_stream()
    x = torch.zeros(20, 256, device="cuda")
    A, W = fp8.quantize_rows(x), fp8.quantize_weight(x.view(2, 10, 256))[0]
    off = torch.tensor([0, 5, 20], dtype=torch.int32, device="cuda")
    r = experts.sort(torch.zeros(10, 2, dtype=torch.int32, device="cuda"), 3)
    w, y = torch.zeros(10, 2, device="cuda"), torch.zeros(10, 256, device="cuda")
    torch.cuda.synchronize()
    for call in (lambda: fp8.quantize_rows(x, index=torch.zeros(20, dtype=torch.int32), stream=side),
                 lambda: fp8.quantize_both(x, offsets=off.cpu(), stream=side),
                 lambda: fp8.product(A, A, C=torch.zeros(20, 20), stream=side),
                 lambda: fp8.product(A, A, out_dtype="f32", beta=1.0, C0=torch.zeros(20, 20), stream=side),
                 lambda: fp8.grouped_product(A, W, off.cpu(), stream=side),
                 lambda: fp8.grouped_product(A, W, off, C=torch.zeros(20, 10), stream=side),
                 lambda: experts.gather(y, r, out=torch.zeros(20, 256), stream=side),
                 lambda: experts.combine(x, r, w, out=torch.zeros(10, 256), stream=side),
                 lambda: experts.combine_gradient(y, x, r, w, dh=torch.zeros(20, 256), stream=side)):
        with pytest.raises(ValueError):
            call()
        assert torch.cuda.current_stream() == before
    side.synchronize()
