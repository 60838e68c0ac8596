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


@pytest.mark.parametrize("T,C", [(5000000, 8), ((1 << 26) + 5000, 1), (9000000, 514)])
def test_routing_of_many_tokens(T, C):
    """More tokens than a launch of a workgroup for each, or for four of them, holds."""
    experts = pytest.importorskip("paper_2506_11209_amd.experts")
    log("case many tokens %d x %d" % (T, C))
    E = 3
    g = torch.Generator(device="cuda").manual_seed(T)
    ids = torch.randint(-1, E, (T, 1), generator=g, device="cuda", dtype=torch.int32)
    r = experts.sort(ids, E)
    n, place = int(r.offsets[-1]), r.place.flatten().long()
    there = place >= 0
    assert n == int(there.sum()) and torch.equal(there, ids.flatten() >= 0)
    x = torch.randn(T, C, generator=g, device="cuda").bfloat16()
    w = torch.randint(1, 5, (T, 1), generator=g, device="cuda").float()
    xs = experts.gather(x, r)
    assert torch.equal(xs[place[there]], x[there]) and (xs[n:] == 0).all()
    y = experts.combine(xs, r, w)
    scaled = (x.float() * w).bfloat16()
    assert torch.equal(y[there], scaled[there]) and (y[~there] == 0).all()
    dh, dw = experts.combine_gradient(x, xs, r, w)
    assert torch.equal(dh[place[there]], scaled[there]) and (dh[n:] == 0).all()
    want = torch.where(there, x.double().square().sum(1), 0.0)
    assert ((dw.flatten().double() - want).abs() <= (C + 1) * 2.0 ** -24 * want).all()


@pytest.mark.parametrize("gathered", (False, True))
def test_quantize_many_rows(gathered):
    """More rows than one launch holds, 32 a workgroup: the same as a part of them by
    itself."""
    R, C = (1 << 29) + 70000, 16
    log("case quantize %d x %d %s" % (R, C, gathered))
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(1000 if gathered else R, C, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    index = torch.randint(-1, 1000, (R,), generator=g, device="cuda", dtype=torch.int32) if gathered else None
    q = fp8.Fp8Matrix.empty(R, C)
    q.codes.view(torch.uint8).fill_(0x7f)
    q.scales.view(torch.uint8).fill_(0xff)
    assert fp8.quantize_rows(x, index=index, out=q) is q
    assert not (q.codes.view(torch.uint8) == 0x7f).any() and not (q.scales.view(torch.uint8) == 0xff).any()  # all of it is written
    for at in (0, (1 << 29) - 33000, R - 70000):
        part = slice(at, at + 70000)
        want = fp8.quantize_rows(x, index=index[part].contiguous()) if gathered else fp8.quantize_rows(x[part])
        assert torch.equal(q.codes[part].view(torch.uint8), want.codes.view(torch.uint8))
        assert torch.equal(q.scales[:, part].view(torch.uint8), want.scales.view(torch.uint8))
