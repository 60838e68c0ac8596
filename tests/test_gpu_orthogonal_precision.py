"""Orthogonalised updates against the iteration in 64 bits, held to what the operator
promises, for matrices whose directions are alike, fall off, or stand out over a weak rest
(as those of gradients do).

Short sides up to 64, up to six steps: the iteration is in binary64; Q and its product with
G are in binary32, which rounds by 2^-24 of Q's largest values, 3.4445^steps, next to a
result of values near 1, two or three times: 1e-4 for five steps (3 * 485 * 2^-24 = 9e-5),
4e-4 for six."""
import pytest
import torch

from tests import orthogonal_ref as ref
from tests.gpu_helpers import log

orthogonal = pytest.importorskip("paper_2506_11209_amd.orthogonal")

pytestmark = pytest.mark.gpu

NAMES = ("noise", "falling", "inverse", "one 0.1", "one 0.00333", "one 0.001", "eighth 0.001", "half 0.01", "rank 2")


def check(G, steps, own):
    got = orthogonal.orthogonalize(G.cuda(), steps).cpu()
    ok, off, bound = ref.within(got, ref.orthogonalize(G, steps), own)
    assert ok, (off, bound)
    return off, bound


@pytest.mark.parametrize("R,C", [(4, 512), (4, 2048), (16, 512), (16, 2048), (17, 33), (64, 64), (64, 300), (300, 50), (2000, 24), (63, 4100), (2, 9)])
@pytest.mark.parametrize("steps", (1, 5, 6))
def test_short_sides(R, C, steps):
    log("case orthogonalize short sides %d x %d, %d steps" % (R, C, steps))
    for i, name in enumerate(NAMES):
        for dtype in (torch.float32, torch.bfloat16, torch.float16):
            G = ref.matrix(R, C, name, seed=i).to(dtype)
            off, bound = check(G, steps, 4e-4 if steps == 6 else 1e-4)
        log("  %-12s off %.2e, bound %.2e" % (name, off, bound))
