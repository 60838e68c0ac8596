"""What the entry points of the 8-bit path and of the routing refuse, and their
sizes on the host: nothing here reaches a GPU."""
import ctypes

import pytest
import torch

from paper_2506_11209_amd import experts, fp8
from paper_2506_11209_amd import wsgemm as w

lib = w.library()
F32, BF16 = w.WS_OUT_F32, w.WS_OUT_BF16
AT = 1 << 20  # an address that is never followed


def matrix(rows=64, cols=256, data=AT, ld=None, dtype=F32, batch=1, stride=0):
    return fp8.ws_matrix(data, rows, cols, cols if ld is None else ld, dtype, batch, stride)


def coded(rows=64, cols=256, codes=AT, scales=AT, ld=None, ld_scales=None, block_rows=1, batch=1, sc=0, ss=0):
    return fp8.ws_fp8_matrix(codes, scales, rows, cols, -(-cols // 16) * 16 if ld is None else ld,
                             -(-rows // block_rows) if ld_scales is None else ld_scales, block_rows, batch, sc, ss)


BAD_MATRIX = [matrix(rows=-1), matrix(cols=-1), matrix(data=0), matrix(data=AT + 2), matrix(ld=255), matrix(dtype=3), matrix(dtype=-1),
              matrix(batch=2, stride=10), matrix(rows=1 << 31)]
BAD_CODED = [coded(codes=0), coded(scales=0), coded(codes=AT + 8), coded(ld=255), coded(ld=264), coded(ld=240), coded(ld_scales=63),
             coded(block_rows=2), coded(rows=-1), coded(batch=-1), coded(batch=2, sc=16), coded(batch=2, sc=64 * 256 + 8, ss=1 << 20)]


def test_quantize_refuses():
    rows, both, weight = lib.ws_fp8_quantize_rows, lib.ws_fp8_quantize_both, lib.ws_fp8_quantize_weight
    for m in BAD_MATRIX:
        assert rows(m, None, coded(), None) == w.WS_ERR_INVALID_ARG
        assert both(m, None, 0, None, coded(), coded(256, 64), None) == w.WS_ERR_INVALID_ARG
        assert weight(m, coded(block_rows=128), None, None) == w.WS_ERR_INVALID_ARG
    for q in BAD_CODED:
        assert rows(matrix(), None, q, None) == w.WS_ERR_INVALID_ARG
        assert both(matrix(), None, 0, None, q, coded(256, 64), None) == w.WS_ERR_INVALID_ARG
    for bad in (coded(65), coded(64, 255), coded(block_rows=128), coded(batch=2, sc=1 << 20, ss=1 << 20)):
        assert rows(matrix(), None, bad, None) == w.WS_ERR_INVALID_ARG
    assert rows(None, None, coded(), None) == w.WS_ERR_INVALID_ARG and rows(matrix(), None, None, None) == w.WS_ERR_INVALID_ARG
    for t in (coded(256, 65), coded(255, 64), coded(256, 64, block_rows=128), coded(256, 128)):
        assert both(matrix(), None, 0, None, coded(), t, None) == w.WS_ERR_INVALID_ARG
    # 64 rows in 3 groups: (64 + 127 * 3) / 128 = 3 blocks
    assert lib.ws_fp8_padded_blocks(64, 3) == 3
    assert both(matrix(), None, 3, AT, coded(), coded(256, 256), None) == w.WS_ERR_INVALID_ARG
    assert both(matrix(), None, 3, None, coded(), coded(256, 384), None) == w.WS_ERR_INVALID_ARG
    assert both(matrix(), None, -1, AT, coded(), coded(256, 64), None) == w.WS_ERR_INVALID_ARG
    ok = coded(block_rows=128)
    for t in (coded(256, 64), coded(64, 256, block_rows=128), coded(256, 64, block_rows=128, batch=2, sc=1 << 20, ss=1 << 20)):
        assert weight(matrix(), ok, t, None) == w.WS_ERR_INVALID_ARG
    assert weight(matrix(), coded(), None, None) == w.WS_ERR_INVALID_ARG


def test_product_refuses():
    f = lib.ws_fp8_product

    def call(A=None, B=None, C=None, C0=None, alpha=1.0, beta=0.0):
        return f(A or coded(), B or coded(32), alpha, beta, C0, C or matrix(64, 32), None)

    for q in BAD_CODED:
        assert call(A=q) == w.WS_ERR_INVALID_ARG and call(B=q) == w.WS_ERR_INVALID_ARG
    for m in BAD_MATRIX:
        assert call(C=m) == w.WS_ERR_INVALID_ARG
    assert call(A=coded(block_rows=128)) == w.WS_ERR_INVALID_ARG
    assert call(A=coded(64, 240)) == w.WS_ERR_INVALID_ARG
    assert call(C=matrix(64, 33)) == w.WS_ERR_INVALID_ARG and call(C=matrix(63, 32)) == w.WS_ERR_INVALID_ARG
    assert call(beta=1.0) == w.WS_ERR_INVALID_ARG
    assert call(beta=1.0, C0=matrix(64, 32, dtype=BF16)) == w.WS_ERR_INVALID_ARG
    assert call(beta=1.0, C0=matrix(64, 31)) == w.WS_ERR_INVALID_ARG
    for bad in (float("nan"), float("inf")):
        assert call(alpha=bad) == w.WS_ERR_INVALID_ARG and call(beta=bad, C0=matrix(64, 32)) == w.WS_ERR_INVALID_ARG
    assert call(A=coded(ld=(1 << 22) + 16)) == w.WS_ERR_INVALID_ARG  # rows too far apart
    assert f(None, coded(32), 1.0, 0.0, None, matrix(64, 32), None) == w.WS_ERR_INVALID_ARG


def test_grouped_products_refuse():
    weights = lambda g, **k: coded(32, block_rows=128, batch=g, sc=32 * 256, ss=2, **k)  # noqa: E731
    f = lib.ws_fp8_grouped_product
    assert f(coded(), weights(3), 2, AT, 1.0, matrix(64, 32), None) == w.WS_ERR_INVALID_ARG
    assert f(coded(), weights(3), 3, None, 1.0, matrix(64, 32), None) == w.WS_ERR_INVALID_ARG
    assert f(coded(), weights(3), 3, AT + 2, 1.0, matrix(64, 32), None) == w.WS_ERR_INVALID_ARG
    assert f(coded(), weights(3), 0, AT, 1.0, matrix(64, 32), None) == w.WS_ERR_INVALID_ARG
    assert f(coded(), weights(3), 3, AT, float("nan"), matrix(64, 32), None) == w.WS_ERR_INVALID_ARG
    assert f(coded(), weights(3), 3, AT, 1.0, matrix(64, 32, batch=3, stride=1 << 20), None) == w.WS_ERR_INVALID_ARG
    g = lib.ws_fp8_grouped_gradient
    a, b, c = coded(64, 384), coded(32, 384), matrix(64, 32, batch=3, stride=64 * 32)
    assert g(a, b, 65, 4, AT, 1.0, 0.0, None, c, None) == w.WS_ERR_INVALID_ARG       # 4 groups: another width
    assert g(a, b, 64, 3, None, 1.0, 0.0, None, c, None) == w.WS_ERR_INVALID_ARG
    assert g(a, b, -1, 3, AT, 1.0, 0.0, None, c, None) == w.WS_ERR_INVALID_ARG
    assert g(a, b, 64, 3, AT, 1.0, 1.0, None, c, None) == w.WS_ERR_INVALID_ARG       # beta without C0
    assert g(a, b, 64, 3, AT, 1.0, 0.0, None, matrix(64, 32), None) == w.WS_ERR_INVALID_ARG
    assert g(a, coded(32, 384, block_rows=128), 64, 3, AT, 1.0, 0.0, None, c, None) == w.WS_ERR_INVALID_ARG


def test_padded_blocks_hold_any_groups():
    for rows in (0, 1, 2, 127, 128, 129, 1000):
        assert lib.ws_fp8_padded_blocks(rows, 0) == -(-rows // 128)
        for groups in (1, 2, 3, 7, 128, 129, 2000):
            got = lib.ws_fp8_padded_blocks(rows, groups)
            # the worst split: one row in each group, the rest in one of them, or any of that kind
            worst = 0
            for ones in range(0, min(groups, rows) + 1):
                left = rows - ones
                if left and ones == groups:
                    continue
                worst = max(worst, ones + -(-left // 128))
            assert worst <= got, (rows, groups)
    assert lib.ws_fp8_padded_blocks(-1, 2) == -1 and lib.ws_fp8_padded_blocks(5, -2) == -1


def test_sort_refuses():
    s = lib.ws_expert_sort
    assert lib.ws_expert_sort_workspace(100, 2, 0) == -1 and lib.ws_expert_sort_workspace(100, 2, 1025) == -1
    assert lib.ws_expert_sort_workspace(-1, 2, 4) == -1 and lib.ws_expert_sort_workspace(100, 0, 4) == -1
    assert lib.ws_expert_sort_workspace(1 << 30, 2, 4) == -1
    assert lib.ws_expert_sort_workspace(100, 2, 4) == 0
    need = lib.ws_expert_sort_workspace(1 << 20, 8, 64)
    assert 0 < need <= 256 * 64 * 4

    def call(tokens=1 << 20, k=8, experts=64, ids=AT, size=4, offsets=AT, token=AT, place=AT, work=AT, bytes_=need):
        return s(tokens, k, experts, ids, size, offsets, token, place, work, bytes_, None)

    for bad in (dict(tokens=-1), dict(k=0), dict(experts=0), dict(experts=1025), dict(ids=None), dict(size=2), dict(size=8, ids=AT + 4),
                dict(offsets=None), dict(token=None), dict(place=None), dict(work=None), dict(bytes_=need - 1), dict(work=AT + 1)):
        assert call(**bad) == w.WS_ERR_INVALID_ARG, bad


def test_rows_refuse():
    x, out = matrix(8, 64), matrix(16, 64)
    gather, combine, grad = lib.ws_expert_gather, lib.ws_expert_combine, lib.ws_expert_combine_gradient
    for m in BAD_MATRIX:
        assert gather(m, 2, 4, AT, AT, out, None) == w.WS_ERR_INVALID_ARG and gather(x, 2, 4, AT, AT, m, None) == w.WS_ERR_INVALID_ARG
        assert combine(m, 2, AT, AT, x, None) == w.WS_ERR_INVALID_ARG and combine(out, 2, AT, AT, m, None) == w.WS_ERR_INVALID_ARG
        assert grad(m, out, 2, 4, AT, AT, AT, out, AT, None) == w.WS_ERR_INVALID_ARG
        assert grad(x, m, 2, 4, AT, AT, AT, out, AT, None) == w.WS_ERR_INVALID_ARG
    assert gather(x, 2, 4, None, AT, out, None) == w.WS_ERR_INVALID_ARG and gather(x, 2, 4, AT, None, out, None) == w.WS_ERR_INVALID_ARG
    assert gather(x, 0, 4, AT, AT, out, None) == w.WS_ERR_INVALID_ARG and gather(x, 2, 0, AT, AT, out, None) == w.WS_ERR_INVALID_ARG
    assert gather(x, 2, 4, AT, AT, matrix(16, 63), None) == w.WS_ERR_INVALID_ARG
    assert gather(x, 2, 4, AT, AT, matrix(16, 64, dtype=BF16), None) == w.WS_ERR_INVALID_ARG
    assert combine(out, 0, AT, AT, x, None) == w.WS_ERR_INVALID_ARG
    assert combine(out, 2, None, AT, x, None) == w.WS_ERR_INVALID_ARG
    assert combine(out, 2, AT, AT + 1, x, None) == w.WS_ERR_INVALID_ARG
    assert grad(x, None, 2, 4, AT, AT, AT, out, AT, None) == w.WS_ERR_INVALID_ARG
    assert grad(x, out, 2, 0, AT, AT, AT, out, AT, None) == w.WS_ERR_INVALID_ARG
    assert grad(x, out, 2, 4, None, AT, AT, out, AT, None) == w.WS_ERR_INVALID_ARG
    assert grad(x, matrix(17, 64), 2, 4, AT, AT, AT, out, AT, None) == w.WS_ERR_INVALID_ARG


def test_empty_calls_touch_nothing():
    none = fp8.ws_matrix(None, 0, 64, 64, F32, 1, 0)
    q0 = coded(0, 64, codes=None, scales=None)
    assert lib.ws_fp8_quantize_rows(none, None, q0, None) == w.WS_OK
    assert lib.ws_fp8_quantize_both(none, None, 0, None, q0, coded(64, 0, codes=None, scales=None), None) == w.WS_OK
    assert lib.ws_fp8_product(q0, coded(32, 64), 1.0, 0.0, None, fp8.ws_matrix(None, 0, 32, 32, F32, 1, 0), None) == w.WS_OK
    assert lib.ws_expert_gather(none, 2, 4, None, None, none, None) == w.WS_OK
    assert lib.ws_expert_combine(none, 2, None, None, none, None) == w.WS_OK


def test_python_refuses_cpu_tensors_and_wrong_types():
    x = torch.zeros(4, 128)
    for call in (lambda: fp8.quantize_rows(x), lambda: fp8.quantize_both(x), lambda: fp8.quantize_weight(x),
                 lambda: fp8.Fp8Matrix(x.to(torch.float8_e4m3fn), x[:1].to(torch.float8_e4m3fn), 4, 128),
                 lambda: fp8.Fp8Matrix(x, x, 4, 128, block_rows=64),
                 lambda: experts.sort(torch.zeros(4, 2, dtype=torch.int32), 4),
                 lambda: experts.Routes(x, x, x)):
        with pytest.raises(ValueError):
            call()
    assert ctypes.sizeof(fp8.ws_matrix) == 48 and ctypes.sizeof(fp8.ws_fp8_matrix) == 72
