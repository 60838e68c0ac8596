"""Weights in 4 bits against the format's definition, and products with them against
64 bits.

Products: each of K products of a bf16 or f16 value and a code is exact in binary32, the
matrix instruction and the waves' parts add them up with an error of at most one
step (2^-23, for sums that are cut) of the sum of magnitudes for each of the at most
K / 8 + 16 additions on a value's way, f16 scales once more: (K / 8 + 20) 2^-23 |A| |B|.
On integers whose sums stay below 2^24 nothing rounds, and results are the rounded
exact ones to the bit."""
import numpy as np
import pytest
import torch

from tests import fp4_ref as ref
from tests.gpu_helpers import log

fp4 = pytest.importorskip("paper_2506_11209_amd.fp4")

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def spread(shape, seed, dtype=torch.float32):
    """Values over many orders of magnitude, zeros, and values halfway between codes."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    x = torch.where(torch.rand(shape, generator=g) < 0.3, (x * 4).round() / 4, x)
    x = x * torch.exp2(torch.randint(-6, 6, shape[:-1] + (1,), generator=g).float())
    x[torch.rand(shape, generator=g) < 0.05] = 0.0
    return x.to(dtype)


def unpacked(q):
    return ref.unpack(q.codes.cpu().numpy(), q.packed_scales.view(torch.uint8).cpu().numpy(), q.rows, q.cols)


@pytest.mark.parametrize("R,C", [(1, 1), (3, 31), (2, 32), (5, 33), (7, 127), (4, 128), (65, 129), (33, 257), (16, 1000), (130, 4104)])
@pytest.mark.parametrize("name", TYPES)
def test_quantize(R, C, name):
    log("case fp4 quantize %d x %d %s" % (R, C, name))
    w = spread((R, C), R * C, TYPES[name])
    q = fp4.quantize_weight(w.cuda())
    codes, scales = ref.quantize(w.double().numpy())
    got = unpacked(q)
    assert np.array_equal(got[1], scales) and np.array_equal(got[0], codes)
    assert np.array_equal(q.scales.view(torch.uint8).cpu().numpy(), scales[:, : -(-C // 32)])
    want = torch.from_numpy(ref.values(codes, scales, C))
    assert torch.equal(q.dequantize().cpu().double(), want)
    assert torch.equal(q.dequantize("bf16").cpu().double(), want)
    assert q.scales.shape == (R, -(-C // 32))


def test_quantize_every_code_and_tie():
    log("case fp4 ties")
    v = torch.tensor([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 5.999, .2499, .2501, 1.2499, 4.99, 5.01])
    w = torch.cat([v, -v[:11]])[None].repeat(3, 1)
    w = w * torch.tensor([[1.0], [2.0 ** -100], [2.0 ** 90]])
    q = fp4.quantize_weight(w.cuda())
    codes, scales = ref.quantize(w.double().numpy())
    assert np.array_equal(unpacked(q)[0], codes) and (q.scales.view(torch.uint8).cpu().flatten().tolist() == [127, 27, 217])


def test_quantize_ends_of_the_range():
    log("case fp4 range")
    w = torch.zeros(6, 64)
    w[0, 0], w[1, 40], w[2, 3], w[3, 5], w[4, 1] = 3.4e38, 1e-45, float("inf"), float("nan"), -1e-38
    w[4, 32] = -3.0
    q = fp4.quantize_weight(w.cuda())
    codes, scales = ref.quantize(w.double().numpy())
    assert np.array_equal(unpacked(q)[1], scales)
    got, want = q.dequantize().cpu().double().numpy(), ref.values(codes, scales, 64)
    assert np.array_equal(got, want, equal_nan=True) and np.isnan(got[2, :32]).all() and (got[2, 32:] == 0).all()


def test_quantize_batch_and_strides():
    log("case fp4 strides")
    big = spread((4, 40, 300), 3, torch.bfloat16).cuda()
    w = big[1:, 3:36, 1:131]
    q = fp4.quantize_weight(w)
    for i in range(3):
        one = fp4.quantize_weight(w[i].contiguous())
        assert torch.equal(q.codes[i], one.codes) and torch.equal(q.packed_scales[i].view(torch.uint8), one.packed_scales.view(torch.uint8))
    codes = torch.full((3, 3, 2080), 7, dtype=torch.uint8, device="cuda")
    scales = torch.full((3, 3, 132), 9, dtype=torch.uint8, device="cuda").view(fp4.E8M0)
    out = fp4.Fp4Matrix(codes, scales, 33, 130)
    assert fp4.quantize_weight(w, out=out) is out
    assert torch.equal(codes[..., :2048], q.codes) and (codes[..., 2048:] == 7).all()
    assert torch.equal(scales.view(torch.uint8)[..., :128], q.packed_scales.view(torch.uint8)) and (scales.view(torch.uint8)[..., 128:] == 9).all()
    assert torch.equal(out.scales.view(torch.uint8), q.scales.view(torch.uint8)) and q.scales.shape == (3, 33, 5)
    into = torch.full((3, 35, 140), 5.0, device="cuda")
    out.dequantize(out=into[:, 1:34, 3:133])
    assert torch.equal(into[:, 1:34, 3:133], q.dequantize()) and (into[:, 0] == 5).all() and (into[..., :3] == 5).all() and (into[..., 133:] == 5).all()


def integers(shape, seed, most):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g).float()


def weights(N, K, seed, lead=()):
    """Values that 4 bits hold: codes, with scales of 1 and 2."""
    g = torch.Generator().manual_seed(seed)
    c = torch.tensor([0.0, 1, 2, 3, 4, 6, 0.5, 1.5, -1, -2, -3, -4, -6, -0.5, -1.5, 6])
    n = -(-K // 32)
    w = c[torch.randint(0, 16, lead + (N, n, 32), generator=g)] * torch.randint(1, 3, lead + (N, n, 1), generator=g)
    return w.flatten(-2)[..., :K].contiguous()


SHAPES = [(1, 1, 1), (1, 17, 31), (2, 16, 32), (15, 33, 100), (16, 64, 128), (17, 65, 129), (31, 70, 255), (33, 128, 513), (49, 31, 384),
          (64, 48, 640), (65, 129, 1000), (130, 40, 2049), (1, 300, 4104),
          (20, 24600, 300), (33, 24600, 160),  # two and four tiles of rows a workgroup
          (20, 25000, 2600), (1100, 1400, 1300), (2100, 800, 1281)]  # and so with A by operands


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("name", ("bf16", "f16"))
def test_product_of_integers(M, N, K, name):
    log("case fp4 product %d x %d x %d %s" % (M, N, K, name))
    x, w = integers((M, K), M + N, 3), weights(N, K, K)  # sums of multiples of 0.5 below 36 * 4104
    W = fp4.quantize_weight(w.cuda())
    assert torch.equal(W.dequantize().cpu(), w)
    want = (x.double() @ w.double().t()).float()
    for out in TYPES:
        got = fp4.product(x.to(TYPES[name]).cuda(), W, out_dtype=out)
        assert got.dtype == TYPES[out] and torch.equal(got.cpu(), want.to(TYPES[out]))


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("name", ("bf16", "f16"))
def test_product_of_values(M, N, K, name):
    log("case fp4 product of values %d x %d x %d %s" % (M, N, K, name))
    g = torch.Generator().manual_seed(M * N + K)
    x = (torch.randn(M, K, generator=g) * torch.where(torch.rand(K, generator=g) < 0.01, 20.0, 1.0)).to(TYPES[name])
    W = fp4.quantize_weight(spread((N, K), K).cuda())
    w = W.dequantize().cpu().double()
    want, size = x.double() @ w.t(), x.double().abs() @ w.abs().t()
    for out in TYPES:
        step = 0.0 if out == "f32" else torch.finfo(TYPES[out]).eps / 2
        got = fp4.product(x.cuda(), W, out_dtype=out).cpu().double()
        bound = (K / 8 + 20) * 2.0 ** -23 * size
        fits = want.abs() + bound < (65000 if out == "f16" else 3e38)
        assert ((got - want).abs() <= bound * (1 + step) + step * want.abs() + (2.0 ** -25 if out == "f16" else 0))[fits].all()


def groups_of(counts, before=0, after=0):
    off = torch.tensor([0] + list(counts)).cumsum(0) + before
    return off.to(torch.int32), int(off[-1]) + after


@pytest.mark.parametrize("counts,before,after", [((3, 0, 1, 20), 0, 0), ((0, 0), 2, 3), ((40, 70, 0, 5), 1, 0), ((1,) * 30, 0, 17), ((0, 129), 5, 2),
                                                 ((16, 32, 64), 0, 0), ((100, 0, 17, 300), 3, 4)])
@pytest.mark.parametrize("name", ("bf16", "f16"))
@pytest.mark.parametrize("N,K", [(70, 300), (4200, 300), (4200, 2650)])  # the last with A by operands, where groups are large
def test_grouped_product(counts, before, after, name, N, K):
    log("case fp4 grouped %s %d %d %s %d x %d" % (counts, before, after, name, N, K))
    off, M = groups_of(counts, before, after)
    E = len(counts)
    x, w = integers((23, K), 1, 3).to(TYPES[name]), weights(N, K, 2, (E,))
    W = fp4.quantize_weight(w.cuda())
    index = torch.randint(-1, 25, (M,), generator=torch.Generator().manual_seed(3)).to(torch.int32)  # -1, 23 and 24: no row
    rows = torch.where(((index >= 0) & (index < 23))[:, None], x[index.clamp(0, 22).long()], torch.zeros((), dtype=x.dtype))
    want = torch.zeros(M, N)
    for e in range(E):
        lo, hi = int(off[e]), int(off[e + 1])
        want[lo:hi] = (rows[lo:hi].double() @ w[e].double().t()).float()
    got = fp4.grouped_product(x.cuda(), W, off.cuda(), index=index.cuda(), out_dtype="f32")
    assert torch.equal(got.cpu(), want)
    into = torch.full((M, N + 9), 3.0, dtype=TYPES[name], device="cuda")
    fp4.grouped_product(rows.cuda(), W, off.cuda(), C=into[:, 2:N + 2])
    assert torch.equal(into[:, 2:N + 2].cpu(), want.to(TYPES[name])) and (into[:, :2] == 3).all() and (into[:, N + 2:] == 3).all()


def test_product_by_index_and_strides():
    log("case fp4 index")
    x, w = integers((9, 203), 1, 3).bfloat16(), weights(40, 200, 2)
    W = fp4.quantize_weight(w.cuda())
    view = x.cuda()[:, 1:201]  # rows at odd places
    index = torch.tensor([8, 0, -3, 8, 9, 1 << 30, 4], dtype=torch.int32)
    want = torch.zeros(7, 40)
    for i, j in enumerate(index.tolist()):
        if 0 <= j < 9:
            want[i] = x[j, 1:201].float() @ w.t()
    assert torch.equal(fp4.product(view, W, index=index.cuda(), out_dtype="f32").cpu(), want)
    assert torch.equal(fp4.product(view, W, out_dtype="f32").cpu(), x[:, 1:201].float() @ w.t())


def test_masked_places_do_not_reach_results():
    """Rows outside a group or past the last, and columns past the last, may hold NaN and infinities."""
    log("case fp4 nan outside")
    big = torch.full((40, 300), float("nan"), dtype=torch.bfloat16)
    x = integers((20, 130), 4, 3).bfloat16()
    big[5:25, 7:137] = x
    big[4, :], big[25, :] = float("inf"), float("-inf")
    w = weights(33, 130, 5, (2,))
    W = fp4.quantize_weight(w.cuda())
    view = big.cuda()[5:25, 7:137]
    assert torch.equal(fp4.grouped_product(view, W, torch.tensor([0, 3, 20], dtype=torch.int32, device="cuda"), out_dtype="f32").cpu(),
                       torch.cat([x[:3].float() @ w[0].t(), x[3:].float() @ w[1].t()]))
    # a NaN in a row stays in that row
    x[2, 129] = float("nan")
    one = fp4.product(x.cuda(), fp4.quantize_weight(w[0].cuda()))
    assert one[2].isnan().all() and one[:2].isfinite().all() and one[3:].isfinite().all()
    # a block of weights with an infinity is NaN
    w[0, 7, 40] = float("inf")
    one = fp4.product(torch.ones(2, 130, dtype=torch.float16, device="cuda"), fp4.quantize_weight(w[0].cuda()))
    assert one[:, 7].isnan().all() and one[:, :7].isfinite().all() and one[:, 8:].isfinite().all()


def test_scales_past_binary16():
    log("case fp4 scales")
    w = weights(20, 96, 1)
    w[:, :32] *= 2.0 ** 60
    w[:, 32:64] *= 2.0 ** -60
    W = fp4.quantize_weight(w.cuda())
    x = torch.zeros(3, 96)
    x[0, :32], x[1, 32:64], x[2, 64:] = 1, 2, 3
    for t in (torch.bfloat16, torch.float16):
        assert torch.equal(fp4.product(x.to(t).cuda(), W, out_dtype="f32").cpu(), (x.double() @ w.double().t()).float())


def test_nothing():
    log("case fp4 nothing")
    for M, N, K in ((0, 5, 7), (3, 0, 7), (3, 5, 0)):
        W = fp4.quantize_weight(torch.ones(N, K, device="cuda"))
        got = fp4.product(torch.ones(M, K, dtype=torch.bfloat16, device="cuda"), W)
        assert got.shape == (M, N) and (got == 0).all() and W.dequantize().shape == (N, K)
    W = fp4.quantize_weight(torch.ones(0, 5, 7, device="cuda"))
    got = fp4.grouped_product(torch.ones(4, 7, dtype=torch.bfloat16, device="cuda"), W, torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert got.shape == (4, 5) and (got == 0).all()


def test_captured_on_a_stream_and_again():
    log("case fp4 graph")
    w = spread((3, 200, 500), 1)
    x = torch.randn(50, 500, device="cuda").bfloat16()
    off = torch.tensor([0, 10, 10, 50], dtype=torch.int32, device="cuda")
    W = fp4.quantize_weight(w.cuda())
    want = fp4.grouped_product(x, W, off)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = fp4.grouped_product(x, fp4.quantize_weight(w.cuda()), off, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph, at = torch.cuda.CUDAGraph(), w.cuda()
    with torch.cuda.graph(graph):
        out = fp4.grouped_product(x, fp4.quantize_weight(at), off)
        one = fp4.product(x, fp4.quantize_weight(at[1]), out_dtype="f32")
    for i in range(3):
        at.copy_(w * (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        W = fp4.quantize_weight(w.cuda() * (i + 1))
        assert torch.equal(out, fp4.grouped_product(x, W, off))
        assert torch.equal(one, fp4.product(x, fp4.quantize_weight(w[1].cuda() * (i + 1)), out_dtype="f32"))


def test_offsets_beyond_32_bits():
    """Matrices and rows more than 2^31 elements apart."""
    log("case fp4 far apart")
    w, x = spread((3, 40, 200), 5, torch.bfloat16), spread((5, 200), 6, torch.bfloat16).clamp(-4, 4)
    room = torch.empty(3 * 2**30 + 2**16, dtype=torch.bfloat16, device="cuda")
    far = room.as_strided((3, 40, 200), (5 * 2**28, 1000, 1))
    far.copy_(w)
    W, want = fp4.quantize_weight(far), fp4.quantize_weight(w.cuda())
    assert torch.equal(W.codes, want.codes) and torch.equal(W.packed_scales.view(torch.uint8), want.packed_scales.view(torch.uint8))
    back = room.as_strided((3, 40, 200), (5 * 2**28, 300, 1))
    assert torch.equal(W.dequantize(out=back), want.dequantize("bf16"))
    codes = room.view(torch.uint8).as_strided((3,) + want.codes.shape[1:], (5 * 2**29, want.codes.shape[2], 1))
    codes.copy_(want.codes)
    W = fp4.Fp4Matrix(codes, want.packed_scales, 40, 200)
    off = torch.tensor([0, 2, 3, 5], dtype=torch.int32, device="cuda")
    assert torch.equal(fp4.grouped_product(x.cuda(), W, off), fp4.grouped_product(x.cuda(), want, off))
    rows, out = room.as_strided((5, 200), (3 * 2**28, 1)), room.as_strided((5, 40), (3 * 2**28, 1), 4096)
    rows.copy_(x)
    fp4.product(rows, fp4.quantize_weight(w[0].cuda()), C=out)
    assert torch.equal(out, fp4.product(x.cuda(), fp4.quantize_weight(w[0].cuda())))


def test_rows_by_operands_captured_and_at_once():
    """Products that lay their rows out in work memory, replayed beside eager ones and on
    two streams."""
    log("case fp4 work memory")
    W = fp4.quantize_weight(spread((1400, 1300), 7).cuda())
    x = [torch.randn(1100, 1300, device="cuda").bfloat16() for _ in range(2)]
    index = torch.randint(-3, 1103, (1200,), dtype=torch.int32, device="cuda")
    want = [fp4.product(v, W, index=index) for v in x]
    inside = (index >= 0) & (index < 1100)
    assert torch.equal(want[0][inside], fp4.product(x[0], W)[index[inside].long()]) and (want[0][~inside] == 0).all()
    streams = [torch.cuda.Stream() for _ in x]
    torch.cuda.synchronize()
    got = [(i, fp4.product(x[i], W, index=index, stream=streams[i])) for _ in range(3) for i in range(2)]
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i]) for i, y in got)
    graph, at = torch.cuda.CUDAGraph(), x[0].clone()
    with torch.cuda.graph(graph):
        out = fp4.product(at, W, index=index)
    for i in (1, 0, 1):
        at.copy_(x[i])
        graph.replay()
        assert torch.equal(fp4.product(x[1 - i], W, index=index), want[1 - i])
        torch.cuda.synchronize()
        assert torch.equal(out, want[i])


def test_refusals():
    log("case fp4 refusals")
    W, E = fp4.quantize_weight(torch.ones(40, 64, device="cuda")), fp4.quantize_weight(torch.ones(2, 40, 64, device="cuda"))
    x = torch.ones(5, 64, dtype=torch.bfloat16, device="cuda")
    off = torch.tensor([0, 2, 5], dtype=torch.int32, device="cuda")
    for call in (lambda: fp4.product(x.float(), W), lambda: fp4.product(x[:, :63], W), lambda: fp4.product(x.cpu(), W), lambda: fp4.product(x, E),
                 lambda: fp4.grouped_product(x, W, off), lambda: fp4.grouped_product(x, E, off[:2]), lambda: fp4.grouped_product(x, E, off.long()),
                 lambda: fp4.grouped_product(x, E, off.cpu()), lambda: fp4.product(x, W, out_dtype="f64"),
                 lambda: fp4.product(x, W, C=torch.zeros(5, 41, device="cuda")), lambda: fp4.product(x, W, C=torch.zeros(5, 40)),
                 lambda: fp4.product(x, W, index=torch.zeros(5, device="cuda")), lambda: fp4.product(x.t(), W),
                 lambda: fp4.quantize_weight(torch.ones(4, 4)), lambda: fp4.quantize_weight(torch.ones(4, 4, device="cuda").double()),
                 lambda: fp4.quantize_weight(torch.ones(4, 8, device="cuda").t()), lambda: fp4.quantize_weight(torch.ones(41, 64, device="cuda"), out=W),
                 lambda: W.dequantize("f16"), lambda: W.dequantize(out=torch.zeros(40, 65, device="cuda")),
                 lambda: fp4.Fp4Matrix(W.codes[:, :1008], W.packed_scales, 40, 64), lambda: fp4.Fp4Matrix(W.codes, W.packed_scales[:, :60], 40, 64),
                 lambda: fp4.Fp4Matrix(W.codes, W.packed_scales.view(torch.uint8), 40, 64), lambda: fp4.Fp4Matrix(W.codes, W.packed_scales, 49, 64),
                 lambda: fp4.Fp4Matrix(W.codes, W.packed_scales, 40, 129)):
        with pytest.raises(ValueError):
            call()
