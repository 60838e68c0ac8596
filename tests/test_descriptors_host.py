"""Descriptors whose batch is 0, as memory cleared by the caller leaves it: a single
matrix, looked at like any other.  Nothing here reaches a GPU."""
from paper_2506_11209_amd import fp8
from paper_2506_11209_amd import wsgemm as w
from tests.test_fp8_host import AT, coded, lib, matrix

INVALID = w.WS_ERR_INVALID_ARG
PLAIN = [dict(data=0), dict(data=AT + 2), dict(ld=7), dict(dtype=3)]
CODED = [dict(codes=0), dict(scales=0), dict(codes=AT + 8), dict(ld=24)]


def plains(rows, cols):
    return [matrix(rows, cols, batch=0, **bad) for bad in PLAIN]


def codeds(rows, cols, **more):
    return [coded(rows, cols, batch=0, **{**more, **bad}) for bad in CODED]


def test_quantize():
    x, q, t = matrix(64, 256), coded(64, 256), coded(256, 64)
    for bad in plains(64, 256):
        assert lib.ws_fp8_quantize_rows(bad, None, q, None) == INVALID
        assert lib.ws_fp8_quantize_both(bad, None, 0, None, q, t, None) == INVALID
    for bad in codeds(64, 256):
        assert lib.ws_fp8_quantize_rows(x, None, bad, None) == INVALID
        assert lib.ws_fp8_quantize_both(x, None, 0, None, bad, t, None) == INVALID
    for bad in codeds(256, 64):
        assert lib.ws_fp8_quantize_both(x, None, 0, None, q, bad, None) == INVALID


def test_products():
    A, B, C = coded(64, 256), coded(32, 256), matrix(64, 32)
    weights = coded(32, 256, block_rows=128, batch=3, sc=32 * 256, ss=2)
    for bad in codeds(64, 256):
        assert lib.ws_fp8_product(bad, B, 1.0, 0.0, None, C, None) == INVALID
        assert lib.ws_fp8_grouped_product(bad, weights, 3, AT, 1.0, C, None) == INVALID
    for bad in codeds(32, 256):
        assert lib.ws_fp8_product(A, bad, 1.0, 0.0, None, C, None) == INVALID
    for bad in plains(64, 32):
        assert lib.ws_fp8_product(A, B, 1.0, 0.0, None, bad, None) == INVALID
        assert lib.ws_fp8_product(A, B, 1.0, 1.0, bad, C, None) == INVALID
        assert lib.ws_fp8_grouped_product(A, weights, 3, AT, 1.0, bad, None) == INVALID
    # 64 rows in 3 groups: 3 blocks
    U, V, G = coded(64, 384), coded(32, 384), matrix(64, 32, batch=3, stride=64 * 32)
    for bad in codeds(64, 384):
        assert lib.ws_fp8_grouped_gradient(bad, V, 64, 3, AT, 1.0, 0.0, None, G, None) == INVALID
    for bad in codeds(32, 384):
        assert lib.ws_fp8_grouped_gradient(U, bad, 64, 3, AT, 1.0, 0.0, None, G, None) == INVALID
    # where the call takes a batch, 0 is none of the groups' matrices
    assert lib.ws_fp8_grouped_product(A, coded(32, 256, block_rows=128, batch=0), 3, AT, 1.0, C, None) == INVALID
    assert lib.ws_fp8_grouped_gradient(U, V, 64, 3, AT, 1.0, 0.0, None, matrix(64, 32, batch=0), None) == INVALID


def test_routing():
    x, h = matrix(8, 64), matrix(16, 64)
    for bad in plains(8, 64):
        assert lib.ws_expert_gather(bad, 2, 4, AT, AT, h, None) == INVALID
        assert lib.ws_expert_combine(h, 2, AT, AT, bad, None) == INVALID
        assert lib.ws_expert_combine_gradient(bad, h, 2, 4, AT, AT, AT, h, AT, None) == INVALID
    for bad in plains(16, 64):
        assert lib.ws_expert_gather(x, 2, 4, AT, AT, bad, None) == INVALID
        assert lib.ws_expert_combine(bad, 2, AT, AT, x, None) == INVALID
        assert lib.ws_expert_combine_gradient(x, bad, 2, 4, AT, AT, AT, h, AT, None) == INVALID
        assert lib.ws_expert_combine_gradient(x, h, 2, 4, AT, AT, AT, bad, AT, None) == INVALID


def test_an_empty_batch_of_weights_does_nothing():
    none = fp8.ws_matrix(None, 64, 256, 256, w.WS_OUT_F32, 0, 0)
    q, t = coded(64, 256, codes=None, scales=None, block_rows=128, batch=0), coded(256, 64, codes=None, scales=None, block_rows=128, batch=0)
    assert lib.ws_fp8_quantize_weight(none, q, t, None) == w.WS_OK
    assert lib.ws_fp8_quantize_weight(none, coded(64, 256, block_rows=128), None, None) == INVALID
    assert lib.ws_fp8_quantize_weight(matrix(64, 256), q, None, None) == INVALID


def test_misaligned_indices():
    x, q, t = matrix(64, 256), coded(64, 256), coded(256, 64)
    for at in (AT + 1, AT + 2):
        assert lib.ws_fp8_quantize_rows(x, at, q, None) == INVALID
        assert lib.ws_fp8_quantize_both(x, at, 0, None, q, t, None) == INVALID
        assert lib.ws_fp8_quantize_both(x, None, 3, at, q, coded(256, 384), None) == INVALID
