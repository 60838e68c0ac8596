"""Orthogonalised updates against the iteration in 64 bits, held to what the operator
promises, for matrices whose directions are alike, fall off, or stand out over a weak rest
(as those of gradients do).

Short sides up to 64, up to six steps: the iteration is in binary64; Q and its product with
G are in binary32, which rounds by 2^-24 of Q's largest values, 3.4445^steps, next to a
result of values near 1, two or three times: 1e-4 for five steps (3 * 485 * 2^-24 = 9e-5),
4e-4 for six.

Sides up to 384, and more than five steps of any: operands are two binary16 values, products
of both rests are left out, sums are in binary32: a step is off by about 2^-22 |X|, and a
direction's error grows with it, 3.4445 a step at the most, until it has arrived: 1.2e-4
for five steps, taken as 2e-4, and 5e-4 for six; for more the weakest directions here, of
1e-4, are off by 1e4 * 2^-22 = 2.4e-3, all of them in the mean by a quarter: 2e-3, with
as much again for what steps near 1 do.

Longer sides, up to five steps: operands of one binary16 value.  A quarter of the directions
of equal size over a rest of 1/1000 are the worst that a replay of the roundings on the CPU found, 2.3e-3
(400 x 4096): taken as 2.4e-3."""
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


def by_hand(steps):
    return 2e-4 if steps <= 5 else 5e-4 if steps == 6 else 2e-3


@pytest.mark.parametrize("R,C", [(65, 128), (66, 1024), (128, 1024), (300, 100), (256, 512), (384, 384), (200, 4100), (1000, 70)])
@pytest.mark.parametrize("steps", (1, 5, 6, 20, 100))
def test_sides_of_some_hundred(R, C, steps):
    log("case orthogonalize %d x %d, %d steps" % (R, C, steps))
    for i, name in enumerate(NAMES):
        if steps >= 20 and name.startswith("rank"):
            continue  # the rounding of G itself arrives
        dtype = (torch.float32, torch.bfloat16, torch.float16)[i % 3]
        off, bound = check(ref.matrix(R, C, name, seed=i).to(dtype), steps, by_hand(steps))
        log("  %-12s off %.2e, bound %.2e" % (name, off, bound))


@pytest.mark.parametrize("R,C", [(400, 500), (513, 513), (600, 1100), (1100, 600), (500, 2048)])
@pytest.mark.parametrize("steps", (1, 5, 6, 20))
def test_longer_sides(R, C, steps):
    log("case orthogonalize %d x %d, %d steps" % (R, C, steps))
    for i, name in enumerate(("noise", "falling", "one 0.1", "eighth 0.001", "quarter 0.001", "half 0.01")):
        off, bound = check(ref.matrix(R, C, name, seed=i), steps, 2.4e-3 if steps <= 5 else by_hand(steps))
        log("  %-12s off %.2e, bound %.2e" % (name, off, bound))


@pytest.mark.parametrize("R", (16, 40, 64))
@pytest.mark.parametrize("steps", (7, 20, 100))
def test_short_sides_of_many_steps(R, steps):
    """The other way round than up to six."""
    log("case orthogonalize %d x 500, %d steps" % (R, steps))
    for i, name in enumerate(("noise", "inverse", "one 0.1", "eighth 0.001")):
        check(ref.matrix(R, 500, name, seed=i), steps, by_hand(steps))


# matrices x rows x columns: what their launches' tiles are (256 CUs)
BATCHES = [
    (1, 250, 300, 5),   # two values; 64 x 64, long rings
    (40, 250, 300, 5),  # 64 x 64, two stages
    (100, 250, 300, 7),
    (350, 250, 300, 5), # 128 x 128: 1050 and 2100 of them
    (20, 640, 700, 6),
    (80, 520, 520, 6),  # 1200 of 128 x 128, five a side
    (12, 500, 512, 5),  # one value; 64 x 64, two stages
    (48, 600, 700, 5),  # 288 lower tiles of 256 x 256: a round, and 32 in quarters; five 128s a side
    (100, 520, 650, 5), # two rounds and 88 in quarters
    (48, 700, 600, 5),
    (44, 600, 513, 5),  # 264: 8 in quarters
]


@pytest.mark.parametrize("B,R,C,steps", BATCHES)
def test_batches_by_their_tiles(B, R, C, steps):
    """Each matrix as by itself, in other tiles, and some against 64 bits.  Of one value to the
    bit; of two, what lies above the diagonal inside a tile adds the two rests' products up the
    other way round than below it: 2^-23 of A, 2e-5 after five steps, so that of a thousand
    values some ten round to a neighbour, 2^-7 of themselves: 8e-4 in norm."""
    log("case orthogonalize %d of %d x %d, %d steps" % (B, R, C, steps))
    names = ("noise", "inverse", "eighth 0.001", "half 0.01")
    some = torch.stack([ref.matrix(R, C, n, seed=i) for i, n in enumerate(names)])
    g = torch.Generator(device="cuda").manual_seed(B)
    G = torch.randn(B, R, C, device="cuda", generator=g)
    at = torch.linspace(0, B - 1, len(names)).long().unique()
    G[at.cuda()] = some[: len(at)].cuda()
    got = orthogonal.orthogonalize(G, steps)
    for i in range(B):
        one = orthogonal.orthogonalize(G[i], steps)
        if min(R, C) > 384 and steps <= 5:
            assert torch.equal(got[i], one), i
        else:
            assert (got[i].double() - one.double()).norm() <= 8e-4 * one.double().norm(), i
    for i in at.tolist()[:: len(at) - 1 or 1]:
        ok, off, bound = ref.within(got[i].cpu(), ref.orthogonalize(G[i].cpu(), steps), 2.4e-3 if min(R, C) > 384 and steps <= 5 else by_hand(steps))
        assert ok, (i, off, bound)


@pytest.mark.parametrize("B,R,C", [(48, 1024, 1024), (60, 512, 1024), (350, 256, 256), (40, 256, 1024)])
def test_signs_in_batches(B, R, C):
    """One step of entries +-1 / 2^k: X, A and A^2 are exact, and so is all of it but T off its
    diagonal, which one binary16 value rounds by 2^-11, two by 2^-22 (and sums in binary32, of less)."""
    log("case orthogonalize signs %d of %d x %d" % (B, R, C))
    g = torch.Generator().manual_seed(B)
    G = torch.where(torch.rand(B, R, C, generator=g) < 0.5, -1.0, 1.0)
    got = orthogonal.orthogonalize(G.cuda(), 1).double().cpu()
    for i in (0, 1, B // 2, B - 1):
        X = G[i].double() / (R * C) ** 0.5
        M = X @ X.t()
        T = ref.B * M + ref.C * M @ M
        want = ref.A * X + T @ X
        unit = 2.0 ** -11 if R > 384 else 2.0 ** -21
        bound = (2.0 ** -8 * want.abs() + unit * (T - T.diagonal().diag()).abs() @ X.abs()) * (1 + 1e-3) + 1e-5 * X.abs().max()
        assert ((got[i] - want).abs() <= bound).all(), i


@pytest.mark.parametrize("R,C", [(64, 65536), (65536, 20), (100, 65536), (65536, 300)])
def test_longest_sides(R, C):
    """Sums of 65536 products: binary32's of values of both signs grow as their square root."""
    log("case orthogonalize %d x %d" % (R, C))
    for i, name in enumerate(("noise", "eighth 0.001")):
        check(ref.matrix(R, C, name, seed=i), 5, by_hand(5))


def test_many_short_matrices():
    log("case orthogonalize 3000 of 66 x 70 and of 30 x 40")
    for R, C in ((66, 70), (30, 40)):
        G = torch.randn(3000, R, C, generator=torch.Generator().manual_seed(R))
        got = orthogonal.orthogonalize(G.cuda()).cpu()
        for i in (0, 1, 1499, 2998, 2999):
            assert ref.within(got[i], ref.orthogonalize(G[i]), by_hand(5))[0], i
