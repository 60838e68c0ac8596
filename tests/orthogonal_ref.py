"""The orthogonalised update by its definition, in 64 bits on the CPU, matrices of chosen
singular values, and how far a result in bf16 may be off."""
import math

import torch

A, B, C = 3.4445, -4.7750, 2.0315


def orthogonalize(G, steps=5):
    """One matrix (rows x columns, any type) in float64."""
    X = G.double()
    X = X / X.norm()
    tall = X.shape[0] > X.shape[1]
    X = X.t() if tall else X
    for _ in range(steps):
        M = X @ X.t()
        X = A * X + (B * M + C * M @ M) @ X
    return X.t() if tall else X


def spectrum(name, n):
    """Singular values: one direction that stands out, some that do over a weak rest, .."""
    s = torch.ones(n, dtype=torch.float64)
    if name == "falling":
        return torch.logspace(0, -4, n, dtype=torch.float64)
    if name == "inverse":
        return 1 / torch.arange(1, n + 1, dtype=torch.float64)
    if name.startswith("one "):
        s[1:] = float(name[4:])
    elif name.startswith("eighth "):
        s[max(1, n // 8):] = float(name[7:])
    elif name.startswith("quarter "):
        s[max(1, n // 4):] = float(name[8:])
    elif name.startswith("half "):
        s[max(1, n // 2):] = float(name[5:])
    elif name.startswith("rank "):  # the others are nothing but what float32 leaves of them
        s[max(1, n // int(name[5:])):] = 0.0
    return s


def matrix(R, C, name, seed=0):
    """R x C of float32 with these singular values (up to its rounding); "noise": independent values."""
    g = torch.Generator().manual_seed(seed)
    if name == "noise":
        return torch.randn(R, C, generator=g)
    n, m = min(R, C), max(R, C)
    u = torch.linalg.qr(torch.randn(n, n, generator=g, dtype=torch.float64))[0]
    v = torch.linalg.qr(torch.randn(m, n, generator=g, dtype=torch.float64))[0]
    x = (u * spectrum(name, n)) @ v.t()
    return (x.t() if R > C else x).float().contiguous()


def rounding(want):
    """|bf16(want) - want|, Frobenius."""
    return (want.bfloat16().double() - want).norm().item()


def within(got, want, own):
    """Whether a result in bf16 is the rounding of one that is off by at most `own` of |want|
    (Frobenius), and both norms.  The two errors have nothing to do with each other: they add
    in squares, but for 1 / sqrt(values) of that by chance; 8 of it are allowed."""
    off, size = (got.double() - want).norm().item(), want.norm().item()
    bound = math.sqrt(rounding(want) ** 2 + (own * size) ** 2) * (1 + 8 / math.sqrt(want.numel()))
    return off <= bound, off / size, bound / size
