"""Products of small integers under scales of powers of two: every sum is exact in
binary32 in any order, and on the 8-bit matrix instruction too, whose eight
neighbouring products lie within its 13 bits of one another.  So each result, in
16 bits as well, is the exact one rounded once, to the bit; a product left out or
taken twice shows.  Every kernel, in every form that launches it."""
import pytest
import torch

from tests import fp8_ref as ref
from tests.gpu_helpers import log
from tests.test_gpu_fp8_kernels import DENSE, DEPTH, ROWS, SHORT, SPLIT, split, stacked, value

fp8 = pytest.importorskip("paper_2506_11209_amd.fp8")

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def integers(rows, cols, seed, block_rows=1):
    """Codes -4 .. 4 without 0, scales 1/2, 1 or 2: products of up to 64, multiples of
    1/4, so that sums over 2^16 columns fit the 24 bits of binary32; values of f16
    results stay below its largest."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = fp8.Fp8Matrix.empty(rows, cols, block_rows)
    c = torch.randint(1, 5, (rows, cols), generator=g, device="cuda") * (1 - 2 * torch.randint(0, 2, (rows, cols), generator=g, device="cuda"))
    q.codes.copy_(torch.zeros(q.codes.shape, device="cuda").to(torch.float8_e4m3fn))
    q.codes[:, :cols] = c.float().to(torch.float8_e4m3fn)
    q.scales.copy_(torch.randint(126, 129, q.scales.shape, generator=g, device="cuda", dtype=torch.uint8).view(torch.float8_e8m0fnu))
    return q


def same(got, a, b, what):
    want = torch.mm(a, b.t().contiguous())
    assert want.abs().max() * 4 < 2 ** 24 if want.numel() else True
    if got.dtype == torch.float16:
        assert want.abs().max() < 65504
    off = got != want.to(got.dtype)
    assert not off.any(), "%s: %d of %d differ, first at %s" % (what, int(off.sum()), off.numel(), off.nonzero()[0].tolist())


@pytest.mark.parametrize("case", [c for c, _ in DENSE + SPLIT], ids=lambda c: "x".join(map(str, c)))
def test_dense(case):
    M, N, K, t = case
    log("case exact %dx%dx%d %s" % case)
    A, B, W = integers(M, K, 1), integers(N, K, 2), integers(N, K, 3, 128)
    same(fp8.product(A, B, out_dtype=t), value(A), value(B), "rows")
    same(fp8.product(A, W, out_dtype=t), value(A), value(W), "weight")
    if t != "f32":  # the same kernels' other type
        other = {"bf16": "f16", "f16": "bf16"}[t]
        same(fp8.product(A, B, out_dtype=other), value(A), value(B), "rows " + other)


@pytest.mark.parametrize("case", [c for c, _ in ROWS], ids=lambda c: "x".join(map(str, c)))
def test_row_groups(case):
    R, N, K, G, t = case
    log("case exact rows %dx%dx%d in %d %s" % case)
    offsets = split(R, G, R)
    A, W = integers(R, K, 1), stacked([integers(N, K, 10 + g) for g in range(G)], N, K)
    got, a = fp8.grouped_product(A, W, torch.tensor(offsets, dtype=torch.int32, device="cuda"), out_dtype=t), value(A)
    for g, (lo, hi) in enumerate(ref.segments(offsets, R)):
        if hi > lo:
            same(got[lo:hi], a[lo:hi], value(fp8.Fp8Matrix(W.codes[g], W.scales[g], N, K, 128)), "group %d" % g)


@pytest.mark.parametrize("case", [c for c, _ in DEPTH + SHORT], ids=lambda c: "x".join(map(str, c)))
def test_depth_groups(case):
    M, N, R, G, t = case
    log("case exact depth %dx%d over %d rows in %d %s" % case)
    offsets, deep = split(R, G, R), fp8.padded_rows(R, G)
    A, B = integers(M, deep, 1), integers(N, deep, 2)
    got, a, b, at = fp8.grouped_gradient(A, B, R, torch.tensor(offsets, dtype=torch.int32, device="cuda"), out_dtype=t), value(A), value(B), 0
    for g, (lo, hi) in enumerate(ref.segments(offsets, R)):
        n = ref.up(hi - lo, 128)
        same(got[g], a[:, at:at + n].contiguous(), b[:, at:at + n].contiguous(), "group %d" % g)
        at += n


@pytest.mark.parametrize("G", (1, 2, 31, 32, 33, 63, 64, 65, 130))
def test_groups_around_a_wave(G):
    """As many groups as a wave has lanes, one fewer and one more, of like and unlike
    depth: by the order of their depths up to 64, else by their own."""
    M, N, R = 1000, 1000, 40 * G + 700
    log("case exact depth of %d groups" % G)
    assert all(p[2] > 0 for p in fp8.plan(M, N, R, "f32", G, True))
    deep = fp8.padded_rows(R, G)
    A, B = integers(M, deep, 1), integers(N, deep, 2)
    a, b = value(A), value(B)
    for offsets in (split(R, G, G), [R // G * g for g in range(G + 1)], [0] * G + [R]):
        got, at = fp8.grouped_gradient(A, B, R, torch.tensor(offsets, dtype=torch.int32, device="cuda")), 0
        for g, (lo, hi) in enumerate(ref.segments(offsets, R)):
            n = ref.up(hi - lo, 128)
            same(got[g], a[:, at:at + n].contiguous(), b[:, at:at + n].contiguous(), "group %d" % g)
            at += n
