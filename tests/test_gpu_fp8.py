"""Quantisation by blocks, the block-scaled product and its grouped forms against
their definitions in 64 bits."""
import numpy as np
import pytest
import torch

from tests import fp8_ref as ref
from tests.gpu_helpers import log

fp8 = pytest.importorskip("paper_2506_11209_amd.fp8")
w = pytest.importorskip("paper_2506_11209_amd.wsgemm")

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def values(rows, cols, dtype, seed, spread=True):
    """Values over many magnitudes, with zeros and an all-zero block."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g)
    if spread:
        x = x * torch.exp2(torch.randint(-12, 5, (rows, cols), generator=g).float())
        x[torch.rand((rows, cols), generator=g) < 0.05] = 0.0
        x[: min(rows, 200), 128:256] = 0.0
    return x.to(dtype)


def check_quantized(q, x, br):
    codes, scales = ref.quantize(x, br)
    got_codes, got_scales = ref.values(q)
    assert np.array_equal(got_scales, scales)
    assert np.array_equal(got_codes, codes, equal_nan=True)


SHAPES = [(1, 1), (1, 128), (3, 17), (16, 4096), (5, 129), (128, 128), (129, 255), (300, 1000), (200, 385), (257, 72)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_quantize_rows_both_and_weight(rows, cols, dtype):
    log("case quantize %dx%d %s" % (rows, cols, dtype))
    x = values(rows, cols, TYPES[dtype], rows * 7 + cols)
    xd, xn = x.cuda(), ref.f64(x)
    check_quantized(fp8.quantize_rows(xd), xn, 1)
    q, t = fp8.quantize_both(xd)
    check_quantized(q, xn, 1)
    check_quantized(t, xn.T, 1)
    q, t = fp8.quantize_weight(xd)
    check_quantized(q, xn, 128)
    check_quantized(t, xn.T, 128)
    assert fp8.quantize_weight(xd, transposed=False)[1] is None


@pytest.mark.parametrize("rows,cols", [(4096, 2048), (4100, 1030)])
def test_quantize_many_rows(rows, cols):
    log("case quantize deep %dx%d" % (rows, cols))
    x = values(rows, cols, torch.bfloat16, 3)
    check_quantized(fp8.quantize_rows(x.cuda()), ref.f64(x), 1)


def test_quantize_extremes():
    """Subnormals, the largest values, ties, and what is not finite."""
    log("case quantize extremes")
    x = torch.zeros(130, 300)
    x[0, :128] = torch.linspace(-448, 448, 128)
    x[1, :3] = torch.tensor([3.4e38, -1.0, 2.0 ** -126])
    x[2, :4] = torch.tensor([1e-45, -2e-45, 2.0 ** -140, 2.0 ** -133])
    x[3, :5] = torch.tensor([float("nan"), 448.0, float("inf"), -float("inf"), 1.0])
    x[4, 100:140] = 448.0 * 2.0 ** -30
    x[5, :130] = torch.cat([torch.tensor([448.0000305, 26.0]), torch.full((128,), float("nan"))])
    x[6, :64] = torch.arange(64) * 0.5 + 0.25  # ties of the coarser steps
    x[7, :2] = torch.tensor([2.0 ** -127, 2.0 ** -149])
    xd = x.cuda()
    check_quantized(fp8.quantize_rows(xd), x.double().numpy(), 1)
    q, t = fp8.quantize_both(xd)
    check_quantized(q, x.double().numpy(), 1)
    check_quantized(t, x.double().numpy().T, 1)
    q, t = fp8.quantize_weight(xd)
    check_quantized(q, x.double().numpy(), 128)
    check_quantized(t, x.double().numpy().T, 128)


def test_quantize_strides_offsets_and_out():
    """Rows further apart, an unaligned start, results in the caller's memory."""
    log("case quantize strides")
    base = values(70, 403, torch.bfloat16, 9).cuda()
    x = base[3:61, 5:305]
    xn = ref.f64(x)
    check_quantized(fp8.quantize_rows(x), xn, 1)
    room = torch.full((58, 400), 7, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    scales = torch.full((3, 80), 9, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    out = fp8.Fp8Matrix(room[:, :304], scales[:, :58], 58, 300)
    t = fp8.Fp8Matrix.empty(300, 58)
    q, got_t = fp8.quantize_both(x, out=(out, t))
    assert q is out and got_t is t
    check_quantized(q, xn, 1)
    check_quantized(t, xn.T, 1)
    assert (room.view(torch.uint8)[:, 304:] == 7).all() and (scales.view(torch.uint8)[:, 58:] == 9).all()
    check_quantized(fp8.quantize_weight(x)[0], xn, 128)


def test_quantize_gathers_rows():
    log("case quantize gather")
    x = values(50, 200, torch.float16, 4)
    index = torch.tensor([3, 3, 49, -1, 0, 50, 7, 1 << 30] * 20, dtype=torch.int32)
    there = (index >= 0) & (index < 50)
    want = torch.where(there[:, None], x[torch.where(there, index, 0).long()], torch.zeros((), dtype=x.dtype))
    check_quantized(fp8.quantize_rows(x.cuda(), index=index.cuda()), ref.f64(want), 1)
    q, t = fp8.quantize_both(x.cuda(), index=index.cuda())
    check_quantized(q, ref.f64(want), 1)
    check_quantized(t, ref.f64(want).T, 1)


GROUPS = {
    "one": [0, 300],
    "uneven": [0, 1, 1, 130, 258, 258, 300],
    "tail": [0, 0, 127, 255],
    "none": [0, 0, 0],
    "many": [0] + sorted(np.random.default_rng(0).integers(0, 300, 149).tolist()) + [300],
}


@pytest.mark.parametrize("name", sorted(GROUPS))
def test_quantize_groups(name):
    log("case quantize groups %s" % name)
    x = values(300, 140, torch.bfloat16, 5)
    offsets = GROUPS[name]
    q, t = fp8.quantize_both(x.cuda(), offsets=torch.tensor(offsets, dtype=torch.int32, device="cuda"))
    xn = ref.f64(x)
    xn[offsets[-1]:] = 0.0
    check_quantized(q, xn, 1)
    check_quantized(t, ref.padded_transpose(xn, offsets), 1)


def test_quantize_weight_batch():
    log("case quantize weight batch")
    x = torch.stack([values(200, 130, torch.float32, s) for s in range(3)])
    q, t = fp8.quantize_weight(x.cuda())
    for i in range(3):
        one = fp8.Fp8Matrix(q.codes[i], q.scales[i], 200, 130, 128)
        check_quantized(one, x[i].double().numpy(), 128)
        check_quantized(fp8.Fp8Matrix(t.codes[i], t.scales[i], 130, 200, 128), x[i].double().numpy().T, 128)


# -- products ------------------------------------------------------------------------

PRODUCTS = [(1, 16, 128), (1, 1, 1), (1, 1000, 4096), (3, 130, 200), (16, 256, 512), (17, 100, 1000), (33, 64, 144), (64, 513, 2048),
            (65, 128, 256), (100, 100, 100), (128, 128, 384), (200, 300, 129), (256, 256, 1024), (257, 511, 640),
            (300, 1000, 1500), (512, 384, 128), (1000, 520, 272)]


def operands(M, N, K, block, seed, scale=1.0):
    a = values(M, K, torch.float32, seed)
    b = values(N, K, torch.float32, seed + 1) * scale
    A = fp8.quantize_rows(a.cuda())
    B = fp8.quantize_rows(b.cuda()) if block == 1 else fp8.quantize_weight(b.cuda(), transposed=False)[0]
    return A, B


@pytest.mark.parametrize("M,N,K", PRODUCTS)
@pytest.mark.parametrize("block", (1, 128))
def test_product(M, N, K, block):
    for out in ("f32", "bf16") if block == 128 else ("f32", "f16"):
        log("case product %dx%dx%d block %d %s" % (M, N, K, block, out))
        A, B = operands(M, N, K, block, M + N + K)
        a, b = ref.dense(A), ref.dense(B)
        want = a @ b.T
        got = fp8.product(A, B, out_dtype=out)
        assert got.dtype is TYPES[out]
        if out == "f16":
            assert np.abs(want).max() < 65000  # nothing here overflows
        ref.assert_within(ref.f64(got), want, ref.product_bound(a, b, want, TYPES[out]), "product")


@pytest.mark.parametrize("M,N,K", [(7, 40, 256), (130, 200, 300), (520, 260, 128)])
@pytest.mark.parametrize("out", sorted(TYPES))
def test_product_alpha_beta(M, N, K, out):
    log("case alpha beta %dx%dx%d %s" % (M, N, K, out))
    A, B = operands(M, N, K, 1, 2)
    a, b = ref.dense(A), ref.dense(B)
    c0 = torch.randn(M, N, generator=torch.Generator().manual_seed(1)).to(TYPES[out])
    for alpha, beta in ((1.0, 1.0), (0.5, -2.0), (0.0, 1.0), (-1.5, 0.0)):
        want = alpha * (a @ b.T) + beta * ref.f64(c0)
        bound = ref.product_bound(a * abs(alpha), b, want, TYPES[out], extra=abs(beta) * np.abs(ref.f64(c0)))
        C0 = c0.cuda()
        got = fp8.product(A, B, out_dtype=out, alpha=alpha, beta=beta, C0=C0)
        ref.assert_within(ref.f64(got), want, bound, "out of place")
        same = fp8.product(A, B, C=C0, alpha=alpha, beta=beta, C0=C0)  # in place
        assert same is C0 and torch.equal(same, got)


def test_product_is_exact_on_integers():
    """Small integers sum exactly in any order: every element, at sizes of every kernel."""
    for M, N, K in ((1, 257, 1024), (40, 300, 640), (150, 270, 400), (520, 1030, 336)):
        log("case integers %dx%dx%d" % (M, N, K))
        g = torch.Generator().manual_seed(M)
        a, b = torch.randint(-4, 5, (M, K), generator=g).float(), torch.randint(-4, 5, (N, K), generator=g).float()
        a[:, 0], b[:, 0] = 4.0, 4.0
        got = fp8.product(fp8.quantize_rows(a.cuda()), fp8.quantize_rows(b.cuda()), out_dtype="f32")
        assert torch.equal(got.cpu().double(), a.double() @ b.double().T)


def test_product_outside_values_and_nan():
    """What lies beside the operands is not read into the result, NaN codes reach
    exactly their rows and columns, and nothing outside C is written."""
    log("case product outside")
    M, N, K = 70, 90, 208
    a, b = values(M, K, torch.float32, 1), values(N, K, torch.float32, 2)
    a[5, 100], b[7, 3] = float("nan"), float("inf")
    room_a = torch.full((M + 9, 256), 0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    room_b = torch.full((N + 9, 272), 0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    A = fp8.quantize_rows(a.cuda(), out=fp8.Fp8Matrix(room_a[3:3 + M, 16:224], fp8.Fp8Matrix.empty(M, K).scales, M, K))
    B = fp8.quantize_rows(b.cuda(), out=fp8.Fp8Matrix(room_b[2:2 + N, 32:240], fp8.Fp8Matrix.empty(N, K).scales, N, K))
    room = torch.full((M + 2, N + 11), 5.0, device="cuda")
    C = fp8.product(A, B, C=room[1:1 + M, 3:3 + N]).cpu()
    nan = torch.zeros(M, N, dtype=torch.bool)
    nan[5], nan[:, 7] = True, True
    assert torch.equal(C.isnan(), nan)
    room[1:1 + M, 3:3 + N] = 5.0
    assert (room == 5.0).all()


def test_product_of_nothing():
    log("case product of nothing")
    for M, N, K in ((0, 5, 128), (5, 0, 128), (5, 7, 0), (0, 0, 0)):
        A, B = fp8.quantize_rows(torch.zeros(M, K, device="cuda")), fp8.quantize_rows(torch.zeros(N, K, device="cuda"))
        C0 = torch.full((M, N), 3.0, device="cuda")
        assert torch.equal(fp8.product(A, B, out_dtype="f32"), torch.zeros(M, N, device="cuda"))
        assert torch.equal(fp8.product(A, B, out_dtype="f32", beta=2.0, C0=C0), 2.0 * C0)


def test_long_rows_far_apart():
    """Rows of a matrix further apart than 32-bit offsets reach over all its rows."""
    log("case long rows")
    ld, M, N, K = 1 << 22, 600, 40, 256
    room = torch.empty(M * ld, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).view(M, ld)
    a, b = values(M, K, torch.float32, 1), values(N, K, torch.float32, 2)
    A = fp8.quantize_rows(a.cuda(), out=fp8.Fp8Matrix(room[:, :K], fp8.Fp8Matrix.empty(M, K).scales, M, K))
    B = fp8.quantize_rows(b.cuda())
    an, bn = ref.dense(A), ref.dense(B)
    want = an @ bn.T
    ref.assert_within(ref.f64(fp8.product(A, B, out_dtype="f32")), want, ref.product_bound(an, bn, want, torch.float32))
    ref.assert_within(ref.f64(fp8.product(B, A, out_dtype="f32")), want.T, ref.product_bound(bn, an, want.T, torch.float32))


def test_operands_past_32_bits():
    """Rows to quantise, and matrices of a batch, at offsets past 2^32: the same bits
    as close together."""
    log("case far operands")
    x = values(70, 300, torch.bfloat16, 1).cuda()
    far = torch.empty(70 << 26, dtype=torch.bfloat16, device="cuda").view(70, 1 << 26)[:, :300]
    far.copy_(x)
    for got, want in zip((fp8.quantize_rows(far),) + fp8.quantize_both(far) + fp8.quantize_weight(far),
                         (fp8.quantize_rows(x),) + fp8.quantize_both(x) + fp8.quantize_weight(x)):
        assert torch.equal(got.codes.view(torch.uint8), want.codes.view(torch.uint8))
        assert torch.equal(got.scales.view(torch.uint8), want.scales.view(torch.uint8))
    E, N, K = 3, 200, 384
    W, _ = fp8.quantize_weight(values(E * N, K, torch.float32, 2).cuda().view(E, N, K), transposed=False)
    room = torch.empty(E, 1 << 32, dtype=torch.uint8, device="cuda")
    codes = room.as_strided((E, N, K), (1 << 32, K, 1)).view(torch.float8_e4m3fn)
    codes.view(torch.uint8).copy_(W.codes.view(torch.uint8))
    A = fp8.quantize_rows(values(300, K, torch.bfloat16, 3).cuda())
    offsets = torch.tensor([0, 120, 121, 290], dtype=torch.int32, device="cuda")
    got = fp8.grouped_product(A, fp8.Fp8Matrix(codes, W.scales, N, K, 128), offsets)
    assert torch.equal(got, fp8.grouped_product(A, W, offsets))


def test_another_stream_and_a_graph():
    """Enqueued on a stream of the caller's; captured and replayed on new data."""
    log("case stream and graph")
    side = torch.cuda.Stream()
    x, wt = values(200, 384, torch.bfloat16, 1).cuda(), values(300, 384, torch.float32, 2).cuda()
    wq, _ = fp8.quantize_weight(wt)
    torch.cuda.synchronize()
    xq = fp8.quantize_rows(x, stream=side)
    y = fp8.product(xq, wq, stream=side)
    side.synchronize()
    want = fp8.product(fp8.quantize_rows(x), wq)
    assert torch.equal(y, want)
    static_x, static_q, static_y = x.clone(), fp8.Fp8Matrix.empty(200, 384), torch.empty(200, 300, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fp8.product(fp8.quantize_rows(static_x, out=static_q), wq, C=static_y)
    for seed in range(4):
        new = values(200, 384, torch.bfloat16, 10 + seed).cuda()
        static_x.copy_(new)
        graph.replay()
        eager = fp8.product(fp8.quantize_rows(new), wq)
        torch.cuda.synchronize()
        assert torch.equal(static_y, eager)


# -- groups ---------------------------------------------------------------------------


@pytest.mark.parametrize("name", sorted(GROUPS))
@pytest.mark.parametrize("N,K", [(48, 256), (200, 144), (300, 520)])
def test_grouped_product_and_gradient(name, N, K):
    log("case groups %s %dx%d" % (name, N, K))
    offsets = GROUPS[name]
    G, R = len(offsets) - 1, 300
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    x = values(R, K, torch.bfloat16, 1)
    wt = torch.stack([values(N, K, torch.float32, 100 + g) for g in range(G)])
    A, At = fp8.quantize_both(x.cuda(), offsets=off)
    W, _ = fp8.quantize_weight(wt.cuda())
    a = ref.dense(A)
    got = ref.f64(fp8.grouped_product(A, W, off, out_dtype="f32"))
    for g, (lo, hi) in enumerate(ref.segments(offsets, R)):
        b = ref.dense(fp8.Fp8Matrix(W.codes[g], W.scales[g], N, K, 128))
        want = a[lo:hi] @ b.T
        ref.assert_within(got[lo:hi], want, ref.product_bound(a[lo:hi], b, want, torch.float32), "group %d" % g)
    assert (got[offsets[-1]:] == 0).all()

    dy = values(R, N, torch.bfloat16, 2)
    _, Dt = fp8.quantize_both(dy.cuda(), offsets=off)
    d, at = ref.dense(Dt), ref.dense(At)
    c0 = torch.randn(G, N, K, generator=torch.Generator().manual_seed(3)).cuda()
    for beta in (0.0, 1.0):
        got = ref.f64(fp8.grouped_gradient(Dt, At, R, off, beta=beta, C0=c0 if beta else None))
        p = 0
        for g, (lo, hi) in enumerate(ref.segments(offsets, R)):
            n = ref.up(hi - lo, 128)
            u, v = d[:, p:p + n], at[:, p:p + n]
            want = u @ v.T + beta * ref.f64(c0[g])
            ref.assert_within(got[g], want, ref.product_bound(u, v, want, torch.float32, extra=beta * np.abs(ref.f64(c0[g]))),
                              "gradient of group %d" % g)
            p += n


def test_grouped_product_few_rows_of_many_groups():
    log("case groups decode")
    G, N, K, R = 70, 160, 384, 96
    counts = np.random.default_rng(1).multinomial(R - 3, np.random.default_rng(2).dirichlet(np.ones(G) * 0.5))
    offsets = [0] + np.cumsum(counts).tolist()
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    A = fp8.quantize_rows(values(R, K, torch.bfloat16, 1).cuda())
    W, _ = fp8.quantize_weight(torch.stack([values(N, K, torch.float32, g) for g in range(G)]).cuda(), transposed=False)
    got, a = ref.f64(fp8.grouped_product(A, W, off, out_dtype="f32")), ref.dense(A)
    for g, (lo, hi) in enumerate(ref.segments(offsets, R)):
        b = ref.dense(fp8.Fp8Matrix(W.codes[g], W.scales[g], N, K, 128))
        want = a[lo:hi] @ b.T
        ref.assert_within(got[lo:hi], want, ref.product_bound(a[lo:hi], b, want, torch.float32))
    assert (got[offsets[-1]:] == 0).all()


def test_linear_layer_gradients():
    """The three products of a layer against the gradients of its formula on the
    same 8-bit operands, and the loss's differences along a direction."""
    log("case linear layer")
    T, N, K = 200, 136, 264
    x, wt, dy = values(T, K, torch.float32, 1, False), values(N, K, torch.float32, 2, False), values(T, N, torch.float32, 3, False)
    xq, xt = fp8.quantize_both(x.cuda())
    wq, wqt = fp8.quantize_weight(wt.cuda())
    gq, gt = fp8.quantize_both(dy.cuda())
    for got, u, v in ((fp8.product(xq, wq, out_dtype="f32"), xq, wq), (fp8.product(gq, wqt, out_dtype="f32"), gq, wqt),
                      (fp8.product(gt, xt, out_dtype="f32"), gt, xt)):
        a, b = ref.dense(u), ref.dense(v)
        ref.assert_within(ref.f64(got), a @ b.T, ref.product_bound(a, b, a @ b.T, torch.float32))
    # loss = sum(dy * y): its difference along a direction u of w is sum(dw * u).  Each quantised
    # factor is within 2^-4 of its value (relative, or of a subnormal step: 2^-9 / 448 of its
    # block's largest), so the two differ by at most (2 * 2^-4 + 2^-8 + 2^-9) of the magnitudes.
    u = values(N, K, torch.float32, 4, False).double().numpy()
    dw = ref.f64(fp8.product(gt, xt, out_dtype="f32"))
    xd, dyd, wd = x.double().numpy(), dy.double().numpy(), wt.double().numpy()
    h = 2.0 ** -10
    loss = lambda m: (dyd * (xd @ m.T)).sum()  # noqa: E731
    difference = (loss(wd + h * u) - loss(wd - h * u)) / (2 * h)
    size = (np.abs(u) * (np.abs(dyd).T @ np.abs(xd))).sum()
    assert abs((dw * u).sum() - difference) <= 0.132 * size


def test_refusals():
    log("case fp8 refusals")
    x = torch.zeros(20, 256, device="cuda")
    A, B = fp8.quantize_rows(x), fp8.quantize_rows(x[:, :240])
    W, Wt = fp8.quantize_weight(x)
    off = torch.tensor([0, 5, 20], dtype=torch.int32, device="cuda")
    stack = fp8.quantize_weight(torch.zeros(2, 8, 256, device="cuda"))[0]
    _, xt = fp8.quantize_both(x, offsets=off)
    for call in (lambda: fp8.product(A, B), lambda: fp8.product(W, A), lambda: fp8.product(A, stack),
                 lambda: fp8.product(A, A, out_dtype="fp8"), lambda: fp8.product(A, A, beta=1.0),
                 lambda: fp8.product(A, A, C=torch.zeros(20, 21, device="cuda")),
                 lambda: fp8.product(A, A, C=torch.zeros(20, 20, device="cuda").t()[:, :20].expand(20, 20)[::1, ::2]),
                 lambda: fp8.product(A, A, C=torch.zeros(20, 20, dtype=torch.int32, device="cuda")),
                 lambda: fp8.product(A, A, beta=1.0, C0=torch.zeros(20, 20, device="cuda")),  # bf16 result
                 lambda: fp8.grouped_product(A, W, off), lambda: fp8.grouped_product(A, stack, off[:2]),
                 lambda: fp8.grouped_product(A, stack, off.long()), lambda: fp8.grouped_product(A, stack, off.cpu()),
                 lambda: fp8.grouped_gradient(xt, xt, 400, off), lambda: fp8.grouped_gradient(xt, W, 20, off),
                 lambda: fp8.quantize_rows(x.t()), lambda: fp8.quantize_rows(x.double()), lambda: fp8.quantize_rows(x[0]),
                 lambda: fp8.quantize_rows(x, index=torch.zeros(4, device="cuda")),
                 lambda: fp8.quantize_rows(x, out=B), lambda: fp8.quantize_rows(x[:1].expand(20, 256)),
                 lambda: fp8.quantize_both(x, offsets=off[:1]),
                 lambda: fp8.Fp8Matrix(A.codes[:, :250], A.scales, 20, 256), lambda: fp8.Fp8Matrix(A.codes, A.scales[:1], 20, 256),
                 lambda: fp8.Fp8Matrix(A.codes[:, 8:248], A.scales, 20, 240), lambda: fp8.Fp8Matrix(A.codes, A.scales, 20, 256, 128)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(w.WsGemmError):
        fp8.product(A, A, alpha=float("inf"))
