"""Rows that belong to no group, before the first one as well as after the last, as
a process sees them that holds some of the experts and passes their part of the
offsets."""
import numpy as np
import pytest
import torch

from tests import fp8_ref as ref
from tests.gpu_helpers import log
from tests.test_gpu_fp8_kernels import ROWS, check, codes, split, stacked, value

fp8 = pytest.importorskip("paper_2506_11209_amd.fp8")

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}

BOUNDS = {
    "head": [5, 40, 40, 130, 300],
    "head and tail": [129, 130, 258, 259],
    "last row": [299, 300],
    "all head": [300, 300, 300],
    "whole blocks": [128, 256, 256, 300],
    "a row each": list(range(1, 300)),  # as many partly filled tiles as there can be
}


def device_offsets(offsets):
    return torch.tensor(offsets, dtype=torch.int32, device="cuda")


def outside(offsets, rows):
    r = torch.arange(rows, device="cuda")
    return (r < offsets[0]) | (r >= offsets[-1])


@pytest.mark.parametrize("name", sorted(BOUNDS))
@pytest.mark.parametrize("gathered", (False, True))
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_quantize(name, gathered, dtype):
    log("case rows outside quantize %s %s %s" % (name, gathered, dtype))
    offsets, R, C = BOUNDS[name], 300, 140
    g = torch.Generator().manual_seed(len(name))
    x = torch.randn(R, C, generator=g).to(TYPES[dtype])
    index = torch.randint(-1, R, (R,), generator=g, dtype=torch.int32) if gathered else None
    # results in memory that holds something else
    deep = fp8.padded_rows(R, len(offsets) - 1)
    out = fp8.Fp8Matrix.empty(R, C), fp8.Fp8Matrix.empty(C, deep)
    for q in out:
        q.codes.view(torch.uint8).fill_(0x55)
        q.scales.view(torch.uint8).fill_(0x77)
    q, t = fp8.quantize_both(x.cuda(), index=index.cuda() if gathered else None, offsets=device_offsets(offsets), out=out)
    xn = ref.f64(x)
    if gathered:
        xn = np.where((index >= 0).numpy()[:, None], xn[index.clamp(min=0).numpy()], 0.0)
    xn[: offsets[0]] = 0.0
    xn[offsets[-1]:] = 0.0
    for got, want in ((q, xn), (t, ref.padded_transpose(xn, offsets))):
        want_codes, want_scales = ref.quantize(want, 1)
        got_codes, got_scales = ref.values(got)
        assert np.array_equal(got_scales, want_scales) and np.array_equal(got_codes, want_codes)


@pytest.mark.parametrize("name", sorted(BOUNDS))
@pytest.mark.parametrize("N,K", [(48, 256), (300, 520)])
def test_product_and_gradient(name, N, K):
    log("case rows outside product %s %dx%d" % (name, N, K))
    offsets, R = BOUNDS[name], 300
    G, off = len(offsets) - 1, device_offsets(offsets)
    A, a = codes(R, K, 1)
    W = stacked([codes(N, K, 10 + g)[0] for g in range(G)], N, K)
    for out in ("f32", "bf16"):
        C = torch.full((R, N), 7.0, dtype=TYPES[out], device="cuda")
        assert fp8.grouped_product(A, W, off, C=C, alpha=2.0 ** -9) is C
        assert (C[outside(offsets, R)] == 0).all()
        for g, (lo, hi) in enumerate(ref.segments(offsets, R)):
            if hi > lo:
                check(C[lo:hi], a[lo:hi], value(fp8.Fp8Matrix(W.codes[g], W.scales[g], N, K, 128)), 2.0 ** -9, what="group %d" % g)
    deep = fp8.padded_rows(R, G)
    (U, u), (V, v), at = codes(N, deep, 3), codes(40, deep, 4), 0
    got = fp8.grouped_gradient(U, V, R, off, alpha=2.0 ** -9)
    for g, (lo, hi) in enumerate(ref.segments(offsets, R)):
        n = ref.up(hi - lo, 128)
        check(got[g], u[:, at:at + n].contiguous(), v[:, at:at + n].contiguous(), 2.0 ** -9, what="gradient of group %d" % g)
        at += n


@pytest.mark.parametrize("case", [c for c, _ in ROWS], ids=lambda c: "x".join(map(str, c)))
def test_every_kernel(case):
    """All groups but the first, their rows with the result's first ones in no group."""
    R, N, K, G, t = case
    log("case rows outside %dx%dx%d in %d %s" % case)
    offsets = split(R, G, R)[1:]
    off = device_offsets(split(R, G, R))[1:]  # a part of the offsets, as a rank takes it
    A, a = codes(R, K, 1)
    W = stacked([codes(N, K, 10 + g)[0] for g in range(G - 1)], N, K)
    C = torch.full((R, N), 7.0, dtype=TYPES[t], device="cuda")
    fp8.grouped_product(A, W, off, C=C, alpha=2.0 ** -9)
    assert (C[outside(offsets, R)] == 0).all()
    for g, (lo, hi) in enumerate(ref.segments(offsets, R)):
        if hi > lo:
            check(C[lo:hi], a[lo:hi], value(fp8.Fp8Matrix(W.codes[g], W.scales[g], N, K, 128)), 2.0 ** -9, what="group %d" % g)
