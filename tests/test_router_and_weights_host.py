"""Refusals of the router's choice, of weights in 4 bits and of orthogonalised updates, at
the C ABI and in the Python calls.  Nothing here reaches a GPU."""
import pytest
import torch

from paper_2506_11209_amd import experts, fp4, orthogonal
from paper_2506_11209_amd import wsgemm as w
from tests.test_fp8_host import AT, lib, matrix

INVALID = w.WS_ERR_INVALID_ARG
BF16, F16 = w.WS_OUT_BF16, w.WS_OUT_F16
PLAIN = [dict(data=0), dict(data=AT + 1), dict(dtype=7), dict(rows=-1), dict(ld=3)]


def change(descriptor, **more):
    copy = type(descriptor).from_buffer_copy(descriptor)
    for name, value in more.items():
        setattr(copy, name, value)
    return copy


def coded(rows, cols, batch=1, **more):
    across, down = -(-cols // 128), -(-rows // 16)
    return change(fp4.ws_fp4_matrix(AT, AT, rows, cols, 1024 * across, 64 * across, batch, down * 1024 * across, down * 64 * across), **more)


CODED = [dict(codes=0), dict(codes=AT + 8), dict(scales=0), dict(scales=AT + 2), dict(ld=1008), dict(ld=1025), dict(ld_scales=60),
         dict(ld_scales=66), dict(rows=-1), dict(cols=-1), dict(batch=-1)]


def test_choose():
    x = matrix(100, 64)
    need = lib.ws_expert_choose_workspace(100000, 64, 4)
    assert 0 < need <= 257 * 65 * 8 and lib.ws_expert_choose_workspace(10, 64, 4) == 0
    for sizes in ((-1, 64, 4), (10, 0, 1), (10, 1025, 1), (10, 64, 0), (10, 64, 33), (10, 3, 4), (1 << 30, 64, 2), ((1 << 30) + 1, 64, 1)):
        assert lib.ws_expert_choose_workspace(*sizes) == -1, sizes

    def call(x=x, k=4, weights=AT, ids=AT, counts=AT, loss=AT, work=None, bytes_=0):
        return lib.ws_expert_choose(x, k, weights, ids, counts, loss, work, bytes_, None)

    for bad in (dict(k=0), dict(k=65), dict(weights=None), dict(ids=None), dict(counts=None), dict(loss=None), dict(ids=AT + 2),
                dict(weights=AT + 1), dict(counts=AT + 2), dict(loss=AT + 2), dict(x=matrix(100, 64, batch=2, stride=6400)), dict(x=matrix(100, 1025)),
                dict(x=matrix(100000, 64)), dict(x=matrix(100000, 64), work=AT, bytes_=need - 1), dict(x=matrix(100000, 64), work=AT + 4, bytes_=need)):
        assert call(**bad) == INVALID, bad
    for bad in PLAIN:
        assert call(x=change(x, **bad)) == INVALID, bad


def test_choose_gradient():
    x = matrix(100, 64)

    def call(x=x, k=4, dweights=AT, dloss=AT, weights=AT, ids=AT, counts=AT, d=x):
        return lib.ws_expert_choose_gradient(x, k, dweights, dloss, weights, ids, counts, d, None)

    for bad in (dict(k=0), dict(k=33), dict(weights=None), dict(ids=None), dict(counts=None), dict(dweights=AT + 2), dict(dloss=AT + 1),
                dict(counts=AT + 2), dict(d=matrix(99, 64)), dict(d=matrix(100, 63)), dict(d=matrix(100, 64, dtype=BF16)), dict(x=matrix(100, 1025))):
        assert call(**bad) == INVALID, bad
    for bad in PLAIN:
        assert call(x=change(x, **bad)) == INVALID and call(d=change(x, **bad)) == INVALID, bad
    none = matrix(0, 64, data=0)
    assert lib.ws_expert_choose_gradient(none, 4, None, None, None, None, None, none, None) == w.WS_OK


def test_casts():
    x, q = matrix(40, 200), coded(40, 200, ld=2048, ld_scales=128)
    for bad in PLAIN:
        assert lib.ws_fp4_quantize(change(x, **bad), q, None) == INVALID and lib.ws_fp4_dequantize(q, change(x, **bad), None) == INVALID, bad
    for bad in CODED:
        assert lib.ws_fp4_quantize(x, change(q, **bad), None) == INVALID and lib.ws_fp4_dequantize(change(q, **bad), x, None) == INVALID, bad
    for other in (coded(41, 200), coded(40, 199), coded(40, 200, batch=2)):
        assert lib.ws_fp4_quantize(x, other, None) == INVALID and lib.ws_fp4_dequantize(other, x, None) == INVALID
    assert lib.ws_fp4_dequantize(q, matrix(40, 200, dtype=F16), None) == INVALID  # does not hold the values
    for bad in CODED:
        assert lib.ws_fp4_scales(change(q, **bad), AT, 7, 280, None) == INVALID, bad
    assert lib.ws_fp4_scales(q, None, 7, 280, None) == INVALID and lib.ws_fp4_scales(q, AT, 6, 280, None) == INVALID
    assert lib.ws_fp4_scales(coded(40, 200, batch=2), AT, 7, 279, None) == INVALID
    two = matrix(40, 200, batch=2, stride=40 * 200)
    for bad in (dict(stride_codes=3 * 2048 - 16), dict(stride_codes=3 * 2048 + 8), dict(stride_scales=3 * 128 - 4), dict(stride_scales=3 * 128 + 2)):
        assert lib.ws_fp4_quantize(two, coded(40, 200, batch=2, **bad), None) == INVALID, bad
    for none in (matrix(0, 200, data=0), matrix(40, 0, data=0)):
        assert lib.ws_fp4_quantize(none, coded(none.rows, none.cols, codes=0, scales=0), None) == w.WS_OK


def test_products():
    A, B, C = matrix(8, 200, dtype=BF16), coded(40, 200), matrix(8, 40)
    weights = coded(40, 200, batch=3)
    for bad in PLAIN:
        assert lib.ws_fp4_product(change(A, **bad), None, B, C, None, 0, None) == INVALID, bad
        assert lib.ws_fp4_product(A, None, B, change(C, **bad), None, 0, None) == INVALID, bad
        assert lib.ws_fp4_grouped_product(change(A, **bad), None, weights, 3, AT, C, None, 0, None) == INVALID, bad
    for bad in CODED:
        assert lib.ws_fp4_product(A, None, change(B, **bad), C, None, 0, None) == INVALID, bad
        assert lib.ws_fp4_grouped_product(A, None, change(weights, **bad), 3, AT, C, None, 0, None) == INVALID, bad
    for a, b, c in ((matrix(8, 200), B, C), (A, coded(40, 199), C), (A, coded(41, 200), C), (A, B, matrix(9, 40)), (A, weights, C)):
        assert lib.ws_fp4_product(a, None, b, c, None, 0, None) == INVALID
    assert lib.ws_fp4_product(A, AT + 2, B, C, None, 0, None) == INVALID
    for groups, offsets in ((2, AT), (-1, AT), (3, None), (3, AT + 1)):
        assert lib.ws_fp4_grouped_product(A, None, weights, groups, offsets, C, None, 0, None) == INVALID
    # work memory, where there are many loads of A
    need = lib.ws_fp4_product_workspace(256, 8192, 8192, -1)
    many = (matrix(256, 8192, dtype=BF16), None, coded(8192, 8192), matrix(256, 8192))
    assert need == 256 * 8192 * 2 and lib.ws_fp4_product_workspace(8, 40, 200, -1) == 0 and lib.ws_fp4_product_workspace(0, 8192, 8192, -1) == 0
    assert lib.ws_fp4_product_workspace(20, 25000, 2600, -1) == 2 * 21 * 4096 and lib.ws_fp4_product_workspace(33, 24600, 160, -1) == 0
    assert lib.ws_fp4_product_workspace(1100, 1400, 1300, -1) == 18 * 4 * 11 * 4096
    assert lib.ws_fp4_product_workspace(112, 4200, 2650, 3) == (112 + 31 * 5) // 32 * 2 * 21 * 4096
    assert lib.ws_fp4_product_workspace(1 << 30, 1 << 30, 1 << 30, 1 << 20) > 0 and lib.ws_fp4_product_workspace(700, 8192, 8192, 0) == 0
    for work, bytes_ in ((None, 0), (None, need), (AT, need - 1), (AT + 8, need)):
        assert lib.ws_fp4_product(*many, work, bytes_, None) == INVALID
    for sizes in ((-1, 5, 5, -1), (5, -1, 5, -1), (5, 5, -1, -1), (5, 5, 5, -2), ((1 << 30) + 1, 5, 5, -1), (5, 5, 5, (1 << 20) + 1)):
        assert lib.ws_fp4_product_workspace(*sizes) == -1, sizes
    for rows, groups in ((16, -1), (16, 1), (64, 4), (16 << 20, 1 << 20)):
        assert lib.ws_fp4_product_workspace(rows, 1 << 20, 1 << 20, groups) == 0
    # no rows of A: they come by an index, or there are none
    assert lib.ws_fp4_product(matrix(0, 200, dtype=BF16, data=0), None, B, C, None, 0, None) == INVALID
    assert lib.ws_fp4_product(matrix(0, 200, dtype=BF16, data=0), None, B, matrix(0, 40, data=0), None, 0, None) == w.WS_OK


def test_orthogonalize():
    need = lib.ws_orthogonal_workspace(300, 200, 2)
    G, out = matrix(300, 200, batch=2, stride=60000), matrix(300, 200, dtype=BF16, batch=2, stride=60000)
    at = AT + 256 - AT % 256
    assert need > 0 and lib.ws_orthogonal_workspace(0, 5, 1) == 0 and lib.ws_orthogonal_workspace(5, 5, 0) == 0
    for sizes in ((-1, 5, 1), (5, -1, 1), (5, 5, -1), (65537, 5, 1), (5, 65537, 1), (5, 5, 1 << 17), (65536, 65536, 64)):
        assert lib.ws_orthogonal_workspace(*sizes) == -1, sizes

    def call(G=G, steps=5, out=out, work=at, bytes_=need):
        return lib.ws_orthogonalize(G, steps, out, work, bytes_, None)

    for bad in (dict(steps=0), dict(steps=101), dict(work=None), dict(work=at + 16), dict(bytes_=need - 1), dict(out=matrix(300, 200, batch=2, stride=60000)),
                dict(out=matrix(200, 300, dtype=BF16, batch=2, stride=60000)), dict(out=matrix(300, 200, dtype=BF16)),
                dict(G=matrix(300, 200, batch=2, stride=59999))):
        assert call(**bad) == INVALID, bad
    for bad in PLAIN:
        assert call(G=change(G, **bad)) == INVALID and call(out=change(out, **bad)) == INVALID, bad
    none = matrix(0, 200, data=0)
    assert lib.ws_orthogonalize(none, 5, matrix(0, 200, dtype=BF16, data=0), None, 0, None) == w.WS_OK


class OnGpu(torch.Tensor):
    """Stands for a tensor on a GPU."""
    is_cuda = True


def stand_in(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


@pytest.mark.parametrize("k", (0, -1, 9, 33, 1 << 32, (1 << 32) + 4, -(1 << 32) + 4))
def test_choices_that_do_not_fit(k):
    with pytest.raises(ValueError):
        experts.choose(stand_in(6, 8), k)


@pytest.mark.parametrize("steps", (0, -1, 101, 1 << 32, (1 << 32) + 5))
def test_steps_that_do_not_fit(steps):
    with pytest.raises(ValueError):
        orthogonal.orthogonalize(stand_in(6, 8), steps)


def test_tensors_on_the_cpu():
    x = torch.zeros(4, 8)
    for call in (lambda: experts.choose(x, 2), lambda: fp4.quantize_weight(x), lambda: orthogonal.orthogonalize(x),
                 lambda: fp4.Fp4Matrix(torch.zeros(1, 1024, dtype=torch.uint8), torch.zeros(1, 64, dtype=torch.uint8).view(fp4.E8M0), 4, 8)):
        with pytest.raises(ValueError):
            call()


def test_optimizer_refuses():
    p = torch.nn.Parameter(torch.zeros(4, 8))
    for bad in (dict(lr=-1.0), dict(momentum=1.0), dict(momentum=-0.1), dict(steps=0), dict(steps=101), dict(weight_decay=-1.0)):
        with pytest.raises(ValueError):
            orthogonal.OrthogonalMomentum([p], **bad)
    for shape in ((4,), (1, 2, 3, 4)):
        with pytest.raises(ValueError):
            orthogonal.OrthogonalMomentum([torch.nn.Parameter(torch.zeros(shape))])
    optimizer = orthogonal.OrthogonalMomentum([p])
    with pytest.raises(ValueError):
        optimizer.add_param_group({"params": [torch.nn.Parameter(torch.zeros(3))]})
    assert len(optimizer.param_groups) == 1
    optimizer.step()  # nothing has a gradient
