"""The 8-bit path's definitions in 64 bits on the CPU, for tests only; shares
nothing with the library."""
from __future__ import annotations

import numpy as np
import torch

BLOCK = 128


def up(n, m):
    return -(-n // m) * m


def round_e4m3(y):
    """float64 -> nearest e4m3 value (ties to even), |y| <= 448."""
    size = np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6)))
    size = np.where(np.exp2(size) > np.maximum(np.abs(y), 2.0 ** -6), size - 1, size)
    step = np.exp2(size - 3)
    return np.rint(y / step) * step


def quantize(x, br, bc=BLOCK):
    """(values of the codes, padded to 16 columns; scales blocks x row blocks) of a
    2-d array in blocks of br x bc; NaN for what is not finite."""
    x = np.asarray(x, dtype=np.float64)
    R, C = x.shape
    a, b = -(-R // br), -(-C // bc)
    v = np.zeros((a * br, b * bc))
    v[:R, :C] = x
    finite = np.isfinite(v)
    amax = np.where(finite, np.abs(v), 0.0).reshape(a, br, b, bc).max(axis=(1, 3)) if R and C else np.zeros((a, b))
    scale = np.ones_like(amax)
    for i in np.ndindex(*amax.shape):
        if amax[i] > 0:
            e = int(np.floor(np.log2(amax[i] / 448.0))) - 1
            while amax[i] > 448.0 * 2.0 ** e:
                e += 1
            scale[i] = 2.0 ** max(e, -127)
    y = np.where(finite, v, 0.0) / np.repeat(np.repeat(scale, br, 0), bc, 1)
    codes = np.where(finite, round_e4m3(y), np.nan)
    return codes[:R, : up(C, 16)], scale.T


def values(q):
    """An Fp8Matrix's (codes, scales) as float64 arrays; scales over columns and rows."""
    codes = q.codes.cpu().float().double().numpy()
    scales = q.scales.cpu().float().double().numpy()
    return codes, scales


def dense(q):
    """An Fp8Matrix (no batch) as a float64 matrix of its columns."""
    codes, scales = values(q)
    s = np.repeat(scales.T, BLOCK, axis=1)[:, : q.cols]
    if q.block_rows > 1:
        s = np.repeat(s, q.block_rows, axis=0)[: q.rows]
    return codes[:, : q.cols] * s


HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def product_bound(a, b, ref, dtype, extra=0.0):
    """How far a product accumulated in binary32 in any order, each addition within
    an ulp (2^-23), and rounded once to dtype may be from the exact one: K ulps of
    the sum of magnitudes, and the output's half ulp (f16 subnormals: 2^-25).  For
    16-bit results the instruction drops of each of eight products what lies below
    2^-13 of the largest: at most 8 * 2^-13 of the sum of magnitudes."""
    s = np.abs(a) @ np.abs(b).T + extra
    if dtype != torch.float32:
        return product_bound(a, b, ref, torch.float32, extra) + 2.0 ** -10 * s + HALF_ULP[dtype] * np.abs(ref) * 1.01 + (
            2.0 ** -25 if dtype == torch.float16 else 0.0)
    return (a.shape[1] + 2) * 2.0 ** -23 * s + HALF_ULP[dtype] * np.abs(ref) * 1.01


def assert_within(got, ref, bound, what=""):
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == ref.shape, (got.shape, ref.shape)
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), "%s: %d of %d off, worst %.3g against a bound of %.3g" % (
        what, bad.sum(), bad.size, np.abs(got - ref)[bad].max(), np.asarray(bound)[bad].min() if np.ndim(bound) else bound)


def f64(t):
    return t.detach().cpu().float().double().numpy() if t.dtype != torch.float32 else t.detach().cpu().double().numpy()


def segments(offsets, rows):
    """[(lo, hi)] of each group."""
    o = [int(v) for v in offsets]
    return [(o[i], o[i + 1]) for i in range(len(o) - 1)]


def padded_transpose(x, offsets):
    """x^T with every group's rows starting at a multiple of 128 (the library's padded order)."""
    x = np.asarray(x, dtype=np.float64)
    R, G = x.shape[0], len(offsets) - 1
    blocks = (R + 127 * min(G, R)) // 128
    out = np.zeros((blocks * BLOCK, x.shape[1]))
    at = 0
    for lo, hi in segments(offsets, R):
        out[at:at + hi - lo] = x[lo:hi]
        at += up(hi - lo, BLOCK)
    return out.T
