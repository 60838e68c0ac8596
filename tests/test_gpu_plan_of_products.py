"""What a product launches is what its plan says: the launches are read from a
captured graph."""
import ctypes

import pytest
import torch

from tests.gpu_helpers import log
from tests.test_gpu_fp8_kernels import DENSE, ROWS, SPLIT, codes, split, stacked

fp8 = pytest.importorskip("paper_2506_11209_amd.fp8")

pytestmark = pytest.mark.gpu


class dim3(ctypes.Structure):
    _fields_ = [("x", ctypes.c_uint32), ("y", ctypes.c_uint32), ("z", ctypes.c_uint32)]


class kernel_node(ctypes.Structure):
    _fields_ = [("block", dim3), ("extra", ctypes.c_void_p), ("func", ctypes.c_void_p), ("grid", dim3),
                ("params", ctypes.c_void_p), ("lds", ctypes.c_uint32)]


def launches(call):
    """[(workgroups, threads of each)] of the kernels that call enqueues, in order."""
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    hip, raw, n = fp8._lib, ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t()  # the library links HIP
    assert hip.hipGraphGetNodes(raw, None, ctypes.byref(n)) == 0
    nodes = (ctypes.c_void_p * n.value)()
    assert hip.hipGraphGetNodes(raw, nodes, ctypes.byref(n)) == 0
    out = []
    for node in nodes:
        k = kernel_node()
        assert hip.hipGraphKernelNodeGetParams(ctypes.c_void_p(node), ctypes.byref(k)) == 0
        out.append((k.grid.x, k.block.x))
    return out


def expected(parts, N, groups=0):
    """Workgroups of each launch of a plan; None for those that follow from the offsets."""
    units = torch.cuda.get_device_properties(0).multi_processor_count
    out = []
    for tile_m, tile_n, stages, rows, launch in parts:
        extra = min(groups + 2, rows) if groups else 0  # partly filled tiles
        tiles = (rows + (tile_m - 1) * extra) // tile_m if groups else -(-rows // tile_m)
        count = tiles * -(-N // tile_n)
        if stages:  # workgroups that stay: one a CU, or two where LDS has room
            count = min(count, units * (2 if tile_m == 64 or (tile_m, stages) == (128, 2) else 1))
        if launch == len(out):
            out.append(count)
        else:
            out[launch] += count
    return out


@pytest.mark.parametrize("case", [c for c, _ in DENSE + SPLIT], ids=lambda c: "x".join(map(str, c)))
def test_dense(case):
    M, N, K, t = case
    log("case plan %dx%dx%d %s" % case)
    A, B = codes(M, K, 1)[0], codes(N, K, 2)[0]
    C = fp8.product(A, B, out_dtype=t)
    parts = fp8.plan(M, N, K, t)
    got = launches(lambda: fp8.product(A, B, C=C))
    assert [g for g, _ in got] == expected(parts, N)
    for tile_m, tile_n, stages, rows, launch in parts:
        assert not stages or got[launch][1] == 256


@pytest.mark.parametrize("case", [c for c, _ in ROWS], ids=lambda c: "x".join(map(str, c)))
def test_row_groups(case):
    R, N, K, G, t = case
    log("case plan rows %dx%dx%d in %d %s" % case)
    off = torch.tensor(split(R, G, R), dtype=torch.int32, device="cuda")
    A, W = codes(R, K, 1)[0], stacked([codes(N, K, 10 + g)[0] for g in range(G)], N, K)
    C = fp8.grouped_product(A, W, off, out_dtype=t)
    assert [g for g, _ in launches(lambda: fp8.grouped_product(A, W, off, C=C))] == expected(fp8.plan(R, N, K, t, G), N, G)
