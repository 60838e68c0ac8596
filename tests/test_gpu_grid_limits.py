"""Products of few rows or columns on the one side and very many on the other, which
need more tiles than a launch has workgroups of one tile each."""
import pytest
import torch

from tests.gpu_helpers import log
from tests.test_gpu_fp8_kernels import check

fp8 = pytest.importorskip("paper_2506_11209_amd.fp8")

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def random_codes(rows, cols, seed):
    """Codes of every magnitude but NaN under scales of one."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = fp8.Fp8Matrix.empty(rows, cols)
    c = q.codes.view(torch.uint8)
    c.random_(0, 256, generator=g)
    c[(c & 0x7f) == 0x7f] = 0x30
    q.scales.view(torch.uint8).fill_(127)
    return q


@pytest.mark.parametrize("M,N,K", [(8, 80000000, 32), (140000000, 8, 16)])
@pytest.mark.parametrize("out", sorted(TYPES))
def test_product(M, N, K, out):
    log("case many tiles %dx%dx%d %s" % (M, N, K, out))
    A, B = random_codes(M, K, 1), random_codes(N, K, 2)
    C = torch.full((M, N), float("nan"), dtype=TYPES[out], device="cuda")
    fp8.product(A, B, C=C, alpha=2.0 ** -9)
    assert not C.isnan().any()  # all of it is written
    side = 1 if N > M else 0
    for at in (0, max(M, N) // 2 - 77, max(M, N) - 3000):
        part = lambda q, s: q.codes[at:at + 3000].float().double() if s else q.codes.float().double()  # noqa: E731
        check(C.narrow(side, at, 3000), part(A, side == 0), part(B, side == 1), 2.0 ** -9, what="from %d" % at)
