"""Sizes whose tiles do not fit the launch of the kernel that would be cheapest: the
plan names one that can run them (host only)."""
import pytest
import torch  # noqa: F401

from paper_2506_11209_amd import fp8

WORKGROUPS = ((1 << 32) - 1) // 512  # of the kernel without a ring, 512 threads each
TILES = 1 << 31                      # that the workgroups of the others take


def launched(M, N, tile_m, tile_n, stages, groups=0, depth=False):
    parts = groups + 2 if groups and not depth else 0
    tiles_m = (M + (tile_m - 1) * min(parts, M)) // tile_m if parts else -(-M // tile_m)
    return tiles_m * -(-N // tile_n) * (groups if depth else 1)


@pytest.mark.parametrize("M,N,K,groups,depth", [
    (8, 80000000, 32, 0, False), (16, 134217728, 128, 0, False), (1, 1 << 30, 16, 0, False), (1 << 30, 1, 16, 0, False),
    (1, 16 * WORKGROUPS, 128, 0, False), (1, 16 * WORKGROUPS + 1, 128, 0, False), (64, 1 << 28, 64, 0, False),
    (1 << 29, 16, 16, 3, False), (3, 40000000, 16, 5, False), (3, 2000, 100, 1 << 20, True), (1 << 25, 30, 500, 9, True)])
@pytest.mark.parametrize("out", ("bf16", "f32"))
def test_a_kernel_that_fits(M, N, K, groups, depth, out):
    parts = fp8.plan(M, N, K, out, groups, depth)
    assert sum(p[3] for p in parts) == M
    for tile_m, tile_n, stages, rows in (p[:4] for p in parts):
        assert launched(rows, N, tile_m, tile_n, stages, groups, depth) <= (TILES if stages else WORKGROUPS)


def test_more_than_any_launch_holds():
    with pytest.raises(fp8._w.WsGemmError):
        fp8.plan(1 << 30, 1 << 30, 128)
    with pytest.raises(fp8._w.WsGemmError):
        fp8.plan(1 << 20, 1 << 20, 128, "f32", 1 << 20, True)
