"""Batches whose matrices lie inside one another, or are one and the same, are
refused as ValueError, like other strides that the library does not take."""
import pytest
import torch

from tests.gpu_helpers import log

fp8 = pytest.importorskip("paper_2506_11209_amd.fp8")

pytestmark = pytest.mark.gpu


def test_batches_that_overlap():
    log("case overlapping batches")
    w = torch.randn(3, 40, 256, device="cuda")
    q, _ = fp8.quantize_weight(w, transposed=False)
    off = torch.tensor([0, 5, 9, 20], dtype=torch.int32, device="cuda")
    deep = fp8.padded_rows(20, 3)
    A, B = fp8.quantize_rows(torch.randn(40, deep, device="cuda")), fp8.quantize_rows(torch.randn(24, deep, device="cuda"))
    for call in (lambda: fp8.quantize_weight(w[:1].expand(3, 40, 256)), lambda: fp8.quantize_weight(w.transpose(0, 1)),
                 lambda: fp8.grouped_gradient(A, B, 20, off, C=torch.zeros(40, 24, device="cuda").expand(3, 40, 24)),
                 lambda: fp8.grouped_gradient(A, B, 20, off, C=torch.zeros(40, 3, 24, device="cuda").transpose(0, 1)),
                 lambda: fp8.grouped_gradient(A, B, 20, off, beta=1.0, C0=torch.zeros(40, 24, device="cuda").expand(3, 40, 24)),
                 lambda: fp8.Fp8Matrix(q.codes[:1].expand(3, 40, 256), q.scales, 40, 256, 128),
                 lambda: fp8.Fp8Matrix(q.codes, q.scales[:1].expand(3, 2, 1), 40, 256, 128),
                 lambda: fp8.Fp8Matrix(q.codes[0, :1].expand(40, 256), q.scales[0], 40, 256, 128),
                 lambda: fp8.Fp8Matrix(A.codes, A.scales[:1].expand(-(-deep // 128), 40), 40, deep)):
        with pytest.raises(ValueError):
            call()
    # further apart than they have to be, or a single one of any stride
    room = torch.randn(3, 50, 300, device="cuda")
    part, _ = fp8.quantize_weight(room[:, 3:43, 5:261], transposed=False)
    want, _ = fp8.quantize_weight(room[:, 3:43, 5:261].contiguous(), transposed=False)
    assert torch.equal(part.codes.view(torch.uint8), want.codes.view(torch.uint8))
    one, _ = fp8.quantize_weight(w.transpose(0, 1)[:, :1].transpose(0, 1), transposed=False)
    assert torch.equal(one.codes.view(torch.uint8), fp8.quantize_weight(w[:1], transposed=False)[0].codes.view(torch.uint8))
