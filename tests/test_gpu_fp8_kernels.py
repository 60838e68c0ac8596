"""Every kernel of the block-scaled product, in every form that launches it, against
a product in 64 bits.  Sizes are ragged, and such that the library picks each of
its kernels; which one it picks is asked of it."""
import numpy as np
import pytest
import torch

from tests import fp8_ref as ref
from tests.gpu_helpers import log

fp8 = pytest.importorskip("paper_2506_11209_amd.fp8")

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
D16, D32, D64 = (16, 16, 0), (32, 16, 0), (64, 16, 0)
T64, T64D, T128, T128D, T256, T256W = (64, 64, 2), (64, 64, 4), (128, 128, 2), (128, 128, 4), (256, 256, 2), (256, 128, 2)

# (M, N, K, type): launches
DENSE = [
    ((9, 300, 520, "f16"), [D16]), ((72, 40, 40, "bf16"), [D32]), ((40, 40, 40, "f32"), [D64]),
    ((130, 3080, 72, "bf16"), [T64]), ((300, 3080, 72, "f32"), [T64]),
    ((130, 1544, 6000, "bf16"), [T64D]), ((130, 3080, 8200, "f32"), [T64D]),
    ((1030, 2056, 72, "f16"), [T128]), ((776, 4104, 72, "f32"), [T128]),
    ((1030, 2056, 4104, "bf16"), [T128D]),
    ((3080, 4104, 776, "bf16"), [T256]), ((2056, 3080, 1544, "f32"), [T256W]),
    ((4104, 1000, 4100, "f32"), [T128, D16]),
    ((2048, 2048, 1024, "bf16"), [T128]), ((4096, 4096, 256, "bf16"), None), ((8192, 2048, 1024, "f16"), [T256]),
]
# (rows, N, K, groups, type): launches
ROWS = [
    ((40, 40, 40, 5, "bf16"), [D16]), ((40, 72, 200, 2, "f32"), [D32]), ((130, 40, 40, 2, "bf16"), [D64]),
    ((130, 3080, 72, 2, "bf16"), [T64]), ((130, 4104, 300, 2, "f32"), [T64]),
    ((40, 4104, 6000, 2, "bf16"), [T64D]), ((130, 3080, 8200, 2, "f32"), [T64D]),
    ((1030, 2056, 72, 2, "bf16"), [T128]), ((776, 4104, 72, 2, "f32"), [T128]), ((1030, 2056, 4104, 2, "f16"), [T128D]),
    ((3080, 4104, 776, 2, "bf16"), [T256]), ((2056, 3080, 1544, 2, "f32"), [T256W]), ((3080, 1030, 520, 9, "bf16"), None),
]
# (M, N, rows, groups, type): launches
DEPTH = [
    ((9, 40, 300, 3, "f32"), [D16]), ((40, 40, 40, 2, "f32"), [D32]), ((72, 40, 200, 2, "bf16"), [D64]),
    ((72, 776, 520, 5, "bf16"), [T64]), ((40, 2056, 520, 5, "f32"), [T64]),
    ((72, 1544, 12000, 2, "bf16"), [T64D]), ((3080, 130, 12000, 2, "f32"), [T64D]),
    ((72, 4104, 520, 5, "bf16"), [T128]), ((72, 4104, 1030, 5, "f32"), [T128]), ((1030, 1030, 8200, 2, "bf16"), [T128D]),
    ((4104, 520, 4104, 5, "bf16"), [T256]), ((1030, 1030, 8200, 5, "f32"), [T256W]),
]

# Last rows by kernels of their own: in the launch of the tiles, or behind it.
SPLIT = [
    ((2314, 417, 4601, "bf16"), [T64, D16]), ((8219, 104, 4315, "bf16"), [T64, D32]), ((773, 1334, 5271, "f16"), [T64D, D16]),
    ((2102, 474, 6647, "bf16"), [T64D, D64]), ((1543, 2612, 1278, "f16"), [T128, D16]), ((2065, 1994, 1286, "bf16"), [T128, D32]),
    ((2216, 1872, 1328, "bf16"), [T128, D64]), ((1643, 2520, 2705, "bf16"), [T128, T64]), ((1936, 2066, 3344, "bf16"), [T128D, D16]),
    ((1557, 2505, 3362, "f16"), [T128D, D32]), ((3341, 4854, 800, "bf16"), [T256, D16]), ((3603, 4509, 920, "bf16"), [T256, D32]),
    ((1162, 858, 3272, "f32"), [T64, D16]), ((1064, 984, 4347, "f32"), [T64, D64]), ((1168, 837, 7327, "f32"), [T64D, D16]),
    ((1665, 2402, 655, "f32"), [T128, D16]), ((1971, 2142, 939, "f32"), [T128, D64]), ((3080, 2580, 1332, "f32"), [T256W, D16]),
    ((5402, 1469, 1283, "f32"), [T256W, D32]),
]

# Few rows in many groups, most of them empty: bound by the results.
SHORT = [
    ((1000, 400, 50, 20, "f32"), [T128]), ((300, 300, 20, 8, "f32"), [T64]), ((1030, 700, 24, 20, "bf16"), [T128]),
    ((390, 520, 1000, 40, "f32"), [T128]), ((260, 1290, 64, 16, "f16"), [T128]),
]


def launches(*args, **kw):
    return [k[:3] for k in fp8.plan(*args, **kw)]


def test_sizes_reach_every_kernel():
    for (M, N, K, t), want in DENSE:
        assert want is None or launches(M, N, K, t) == want, (M, N, K, t)
    for (R, N, K, g, t), want in ROWS:
        assert want is None or launches(R, N, K, t, g) == want, (R, N, K, g, t)
    for (M, N, R, g, t), want in DEPTH:
        assert want is None or launches(M, N, R, t, g, True) == want, (M, N, R, g, t)
    for cases in (DENSE, ROWS, DEPTH):
        for wide in (False, True):
            seen = {k for c, w in cases if (c[-1] == "f32") == wide for k in w or ()}
            everything = {D16, D32, D64, T64, T64D, T128} | ({T256W} if wide else {T128D, T256})
            assert everything - seen <= {D16, D32, D64}, (cases[0], wide, everything - seen)
    assert fp8.plan(0, 5, 5) == [] and sum(k[3] for k in fp8.plan(4104, 1000, 4100, "f32")) == 4104


def test_few_rows_in_many_groups_run_as_tiles():
    for (M, N, R, g, t), want in SHORT:
        assert launches(M, N, R, t, g, True) == want, (M, N, R, g, t)


def test_last_rows_by_themselves():
    for (M, N, K, t), want in SPLIT:
        assert launches(M, N, K, t) == want, (M, N, K, t)
        assert [k[3] for k in fp8.plan(M, N, K, t)] == [M // 128 * 128, M % 128]


def test_plan_refuses():
    for bad in ((-1, 5, 5), (5, -1, 5), (5, 5, -1), (5, 5, 1 << 31)):
        with pytest.raises(fp8._w.WsGemmError):
            fp8.plan(*bad)
    with pytest.raises(fp8._w.WsGemmError):
        fp8.plan(5, 5, 5, groups=-1)
    with pytest.raises(fp8._w.WsGemmError):
        fp8.plan(5, 5, 5, groups=0, depth=True)
    with pytest.raises(ValueError):
        fp8.plan(5, 5, 5, "fp8")


def codes(rows, cols, seed, spread=3):
    """A matrix of random codes and scales with exact values: (Fp8Matrix, float64 on
    the GPU).  Codes of every magnitude, scales over 2^-spread .. 2^spread."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = fp8.Fp8Matrix.empty(rows, cols)
    c = torch.randint(0, 256, q.codes.shape, generator=g, device="cuda", dtype=torch.uint8)
    c = torch.where((c & 0x7f) == 0x7f, torch.full_like(c, 0x30), c)  # no NaN
    c[:, cols:] = 0
    q.codes.copy_(c.view(torch.float8_e4m3fn))
    s = torch.randint(127 - spread, 128 + spread, q.scales.shape, generator=g, device="cuda", dtype=torch.uint8)
    q.scales.copy_(s.view(torch.float8_e8m0fnu))
    return q, value(q)


def value(q):
    k, n = torch.arange(q.cols, device="cuda") // 128, torch.arange(q.rows, device="cuda") // q.block_rows
    s = q.scales.float().double()
    return q.codes[:, : q.cols].float().double() * s[k][:, n].t()


def check(got, a, b, alpha=1.0, c0=None, beta=0.0, what=""):
    """got against alpha a b^T + beta c0, with the bound of product_bound."""
    want = alpha * torch.mm(a, b.t().contiguous())
    size = abs(alpha) * torch.mm(a.abs(), b.abs().t().contiguous())
    if beta:
        want, size = want + beta * c0.double(), size + abs(beta) * c0.double().abs()
    bound = (a.shape[1] + 2) * 2.0 ** -23 * size + ref.HALF_ULP[got.dtype] * want.abs() * 1.01
    if got.dtype != torch.float32:
        bound = bound + 2.0 ** -10 * size + ref.HALF_ULP[got.dtype] * want.abs() * 1.01 + 2.0 ** -25
    top = 65504.0 if got.dtype == torch.float16 else float("inf")
    fits = want.abs() + bound < top  # f16 overflows to infinity elsewhere
    off = ((got.double() - want).abs() > bound) & fits
    assert not off.any(), "%s: %d of %d off, first at %s" % (what, int(off.sum()), off.numel(), off.nonzero()[0].tolist())
    assert fits.float().mean() > 0.5


@pytest.mark.gpu
@pytest.mark.parametrize("case", [c for c, _ in DENSE + SPLIT], ids=lambda c: "x".join(map(str, c)))
def test_dense(case):
    M, N, K, t = case
    log("case dense %dx%dx%d %s" % case)
    A, a = codes(M, K, 1)
    B, b = codes(N, K, 2)
    check(fp8.product(A, B, out_dtype=t, alpha=2.0 ** -9), a, b, 2.0 ** -9, what="rows")
    c0 = torch.randn(M, N, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(TYPES[t])
    check(fp8.product(A, B, out_dtype=t, alpha=2.0 ** -9, beta=0.5, C0=c0), a, b, 2.0 ** -9, c0, 0.5, "beta")
    # a view of a wider result: unaligned rows
    room = torch.full((M, N + 7), 3.0, dtype=TYPES[t], device="cuda")
    fp8.product(A, B, C=room[:, 3:3 + N], alpha=2.0 ** -9)
    check(room[:, 3:3 + N], a, b, 2.0 ** -9, what="view")
    assert (room[:, :3] == 3).all() and (room[:, 3 + N:] == 3).all()
    # scales for 128 x 128
    W = fp8.Fp8Matrix(B.codes, B.scales[:, : -(-N // 128)].contiguous(), N, K, 128)
    check(fp8.product(A, W, out_dtype=t, alpha=2.0 ** -9), a, value(W), 2.0 ** -9, what="weight")


def split(rows, groups, seed):
    """Offsets: uneven, some groups empty, some rows in none."""
    rng = np.random.default_rng(seed)
    counts = rng.multinomial(rows - rows // 20, rng.dirichlet(np.ones(groups)))
    if groups > 2:
        counts[groups // 2] = 0
    return [0] + np.cumsum(counts).tolist()


def stacked(parts, N, K):
    """A batch with 128 x 128 scales from matrices with row scales."""
    both = [torch.stack([t.view(torch.uint8) for t in ts]) for ts in zip(*((p.codes, p.scales[:, : -(-N // 128)]) for p in parts))]
    return fp8.Fp8Matrix(both[0].view(torch.float8_e4m3fn), both[1].contiguous().view(torch.float8_e8m0fnu), N, K, 128)


@pytest.mark.gpu
@pytest.mark.parametrize("case", [c for c, _ in ROWS], ids=lambda c: "x".join(map(str, c)))
def test_row_groups(case):
    R, N, K, G, t = case
    log("case rows %dx%dx%d in %d %s" % case)
    offsets = split(R, G, R)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    A, a = codes(R, K, 1)
    parts = [codes(N, K, 10 + g)[0] for g in range(G)]
    W = stacked(parts, N, K)
    got = fp8.grouped_product(A, W, off, out_dtype=t, alpha=2.0 ** -9)
    for g, (lo, hi) in enumerate(ref.segments(offsets, R)):
        if hi > lo:
            check(got[lo:hi], a[lo:hi], value(fp8.Fp8Matrix(W.codes[g], W.scales[g], N, K, 128)), 2.0 ** -9, what="group %d" % g)
    assert (got[offsets[-1]:] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("case", [c for c, _ in DEPTH + SHORT], ids=lambda c: "x".join(map(str, c)))
def test_depth_groups(case):
    M, N, R, G, t = case
    log("case depth %dx%d over %d rows in %d %s" % case)
    offsets = split(R, G, R)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    deep = fp8.padded_rows(R, G)
    A, a = codes(M, deep, 1)
    B, b = codes(N, deep, 2)
    c0 = torch.randn(G, M, N, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(TYPES[t])
    for beta in (0.0, 0.5):
        got = fp8.grouped_gradient(A, B, R, off, out_dtype=t, alpha=2.0 ** -9, beta=beta, C0=c0 if beta else None)
        at = 0
        for g, (lo, hi) in enumerate(ref.segments(offsets, R)):
            n = ref.up(hi - lo, 128)
            check(got[g], a[:, at:at + n].contiguous(), b[:, at:at + n].contiguous(), 2.0 ** -9, c0[g], beta, "group %d" % g)
            at += n


@pytest.mark.gpu
def test_offsets_out_of_order_stay_inside():
    """Offsets that decrease or leave the rows are cut to them: the result's rows
    outside are zeros, nothing else is promised but that memory beside is untouched."""
    log("case offsets out of order")
    R, N, K, G = 200, 100, 256, 4
    A, _ = codes(R, K, 1)
    parts = [codes(N, K, 10 + g)[0] for g in range(G)]
    W = stacked(parts, N, K)
    for offsets in ([0, 500, 100, -7, 200], [-50, 20, 20, 1 << 30, 1 << 30], [200, 100, 50, 20, 0]):
        off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        room = torch.full((R + 2, N), 3.0, dtype=torch.bfloat16, device="cuda")
        fp8.grouped_product(A, W, off, C=room[1:1 + R])
        deep = fp8.padded_rows(R, G)
        u, v = codes(40, deep, 1)[0], codes(30, deep, 2)[0]
        fp8.grouped_gradient(u, v, R, off)
        fp8.quantize_both(torch.randn(R, 50, device="cuda"), offsets=off)
        torch.cuda.synchronize()
        assert (room[0] == 3).all() and (room[-1] == 3).all()


@pytest.mark.gpu
@pytest.mark.parametrize("case,ld", [((4104, 1000, 4100, "f32"), 1 << 20), ((1543, 2612, 1278, "f16"), 1 << 22),
                                     ((3341, 4854, 800, "bf16"), 1 << 20), ((9, 300, 520, "bf16"), 1 << 29)], ids=str)
def test_results_past_32_bits(case, ld):
    """Rows of C so far apart that offsets pass 2^32: the same bits as dense."""
    M, N, K, t = case
    log("case far results %s %d" % (case, ld))
    A, B = codes(M, K, 1)[0], codes(N, K, 2)[0]
    room = torch.empty(M * ld, dtype=TYPES[t], device="cuda").view(M, ld)
    room[:, N:N + 8] = 3.0
    C = fp8.product(A, B, C=room[:, :N], alpha=2.0 ** -9)
    assert torch.equal(C, fp8.product(A, B, out_dtype=t, alpha=2.0 ** -9)) and (room[:, N:N + 8] == 3.0).all()
    if t == "f32":
        fp8.product(A, B, C=C, alpha=2.0 ** -9, beta=-1.0, C0=C)  # in place: the same sums, so exactly zero
        assert (C == 0).all()
