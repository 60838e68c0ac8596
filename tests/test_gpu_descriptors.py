"""A descriptor whose batch is 0 stands for a single matrix, as batch 1 does."""
import pytest
import torch

from tests.gpu_helpers import log

fp8 = pytest.importorskip("paper_2506_11209_amd.fp8")
experts = pytest.importorskip("paper_2506_11209_amd.experts")

pytestmark = pytest.mark.gpu


def test_batch_0_is_a_single_matrix():
    log("case batch 0")
    lib = fp8._lib
    x, y = torch.randn(40, 256, device="cuda"), torch.randn(24, 256, device="cuda")
    want_q = fp8.quantize_rows(x)
    q, other = fp8.Fp8Matrix.empty(40, 256), fp8.quantize_rows(y)
    want = fp8.product(want_q, other, out_dtype="f32")
    C = torch.zeros_like(want)
    mx, mc = fp8._matrix(x, "x"), fp8._matrix(C, "C")
    for desc in (mx, mc, q._desc, other._desc):
        desc.batch = 0
    assert lib.ws_fp8_quantize_rows(mx, None, q._desc, None) == 0
    assert torch.equal(q.codes.view(torch.uint8), want_q.codes.view(torch.uint8))
    assert torch.equal(q.scales.view(torch.uint8), want_q.scales.view(torch.uint8))
    assert lib.ws_fp8_product(q._desc, other._desc, 1.0, 0.0, None, mc, None) == 0
    assert torch.equal(C, want)
    r = experts.sort(torch.arange(40, dtype=torch.int32, device="cuda").view(40, 1) % 7, 7)
    out = torch.zeros_like(x)
    mo = fp8._matrix(out, "out")
    mo.batch = 0
    assert lib.ws_expert_gather(mx, 1, 7, r.offsets.data_ptr(), r.place.data_ptr(), mo, None) == 0
    assert torch.equal(out, experts.gather(x, r))
