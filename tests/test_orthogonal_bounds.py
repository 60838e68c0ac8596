"""What the bound of tests/orthogonal_ref.py tells apart, on the CPU: the iteration in 32
bits passes it; zeros, a step too few or too many, another coefficient, and the errors that
binary32's Gram matrix of six steps and operands in binary16 leave do not."""
import pytest
import torch

from tests import orthogonal_ref as ref


def binary32(G, steps):
    X = G.float() / G.double().norm().float()
    for _ in range(steps):
        M = X @ X.t()
        X = ref.A * X + (ref.B * M + ref.C * M @ M) @ X
    return X.bfloat16()


@pytest.mark.parametrize("R,C", [(4, 512), (17, 33), (65, 128), (64, 300), (128, 1024)])
@pytest.mark.parametrize("name", ("noise", "falling", "inverse", "one 0.001", "eighth 0.001", "half 0.01"))
@pytest.mark.parametrize("steps", (5, 6))
def test_tells_apart(R, C, name, steps):
    G = ref.matrix(R, C, name)
    want = ref.orthogonalize(G, steps)
    assert ref.within(binary32(G, steps), want, 1e-4)[0]
    assert ref.within(want.bfloat16(), want, 0.0)[0]
    for wrong in (torch.zeros(R, C), ref.orthogonalize(G, steps - 1), ref.orthogonalize(G, steps + 1), want * 1.01, -want):
        assert not ref.within(wrong.bfloat16(), want, 2e-3)[0]


def test_gram_matrix_in_binary32():
    """Six steps by way of A alone, as A <- T A T in binary32."""
    G = ref.matrix(4, 512, "one 0.001")
    X = G.float() / G.norm()
    M, Q = X @ X.t(), torch.eye(4)
    for _ in range(6):
        T = ref.A * torch.eye(4) + ref.B * M + ref.C * M @ M
        Q, M = T @ Q, T @ M @ T
    assert not ref.within((Q @ X).bfloat16(), ref.orthogonalize(G, 6), 1e-3)[0]


def test_operands_in_binary16():
    G = ref.matrix(66, 512, "eighth 0.001")
    X = G.double() / G.double().norm()
    for _ in range(5):
        H = (X * 2.0 ** 14).half().double() / 2.0 ** 14
        M = H @ H.t()
        d = M.diagonal()
        M = ((M - d.diag()) * 2.0 ** 14).half().double() / 2.0 ** 14 + d.diag()
        T = ref.B * M + ref.C * M @ M
        d = T.diagonal()
        T = ((T - d.diag()) * 2.0 ** 14).half().double() / 2.0 ** 14
        X = ref.A * X + d[:, None] * X + T @ H
    want = ref.orthogonalize(G)
    ok, off, bound = ref.within(X.bfloat16(), want, 1e-4)
    assert not ok and off > 2e-3
