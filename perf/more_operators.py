"""Operators beside a layer of experts: the router's choice with its balance loss and
gradient, the orthogonalised update of weights, and products with weights in 4 bits.

Each case is one pass through the public Python entry points (``own`` true:
``paper_2506_11209_amd.experts``, ``.orthogonal`` and ``.fp4``) or through the plain
form of the same operator in elementary torch operations (``own`` false).

The choice: for logits l (tokens x experts), ids are each token's k largest (the
lowest index first among equals; a logit of -inf is never chosen, -1 stands in its
place), weights their softmax, counts[e] the choices of expert e and counts[experts]
the tokens that have any; loss = experts * sum_e counts[e] / choices * mean_t p_te,
p the softmax over all experts, the mean over the tokens that have a choice.

The orthogonalised update: X = G / |G| (Frobenius), then X <- a X + (b A + c A^2) X
with A = X X^T, five times; results in bf16.

4-bit weights: codes are e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), a
scale is a power of two in 8 bits for 32 columns of a row, the smallest s with the
block's largest magnitude at most 6 s; codes round to nearest, ties to even.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 32  # columns of a row that share a scale in 4 bits
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
A1, A3, A5 = 3.4445, -4.7750, 2.0315
STEPS = 5


# -- cases ------------------------------------------------------------------------


def listed():
    return [
        # A decoding batch through the router: latency.
        {"name": "choose_32x64", "kind": "choose", "T": 32, "E": 64, "k": 4, "type": "f32", "masked": 0.0},
        # A large training batch over many experts, some of its tokens padding.
        {"name": "choose_65536x256", "kind": "choose", "T": 65536, "E": 256, "k": 8, "type": "bf16", "masked": 0.05},
        # The way back of a training step's choice.
        {"name": "choose_gradient_8192x64", "kind": "choose_gradient", "T": 8192, "E": 64, "k": 4, "type": "f32", "masked": 0.02},
        # The same for odd sizes.
        {"name": "choose_gradient_30001x100", "kind": "choose_gradient", "T": 30001, "E": 100, "k": 2, "type": "bf16", "masked": 0.02},
        # The router's own update: a few long rows, latency.
        {"name": "orthogonalize_16x2048", "kind": "orthogonalize", "B": 1, "R": 16, "C": 2048, "type": "f32"},
        # One matrix of ragged sizes, taller than wide.
        {"name": "orthogonalize_2500x1000", "kind": "orthogonalize", "B": 1, "R": 2500, "C": 1000, "type": "bf16"},
        # The weight gradients of a layer of 16 experts.
        {"name": "orthogonalize_16of4096x2048", "kind": "orthogonalize", "B": 16, "R": 4096, "C": 2048, "type": "f32"},
        # A weight rounded to 4 bits and back, as training for 4 bits does each step.
        {"name": "quantize_4100x4104", "kind": "quantize", "B": 1, "R": 4100, "C": 4104, "type": "f32"},
        # The experts of a layer, rounded for serving.
        {"name": "quantize_16of4096x2048", "kind": "quantize", "B": 16, "R": 4096, "C": 2048, "type": "bf16"},
        # One token through a linear layer.
        {"name": "product_1x8192x8192", "kind": "product", "M": 1, "N": 8192, "K": 8192, "type": "bf16", "out": "bf16"},
        # A batch of tokens that fills no tile, ragged sizes, results in 32 bits.
        {"name": "product_40x4104x4100", "kind": "product", "M": 40, "N": 4104, "K": 4100, "type": "f16", "out": "f32"},
        # A decoding batch of 32 tokens, four experts of 64 each: a few rows, some none.
        {"name": "grouped_decode_32of64", "kind": "grouped", "T": 32, "k": 4, "E": 64, "N": 4096, "K": 2048, "type": "bf16",
         "out": "bf16", "masked": 0.0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("choose", "choose", "choose_gradient", "choose_gradient", "orthogonalize", "orthogonalize", "orthogonalize",
                       "quantize", "product", "product", "grouped"))
    typ = rng.choice(("bf16", "f16", "f32"))
    if kind in ("choose", "choose_gradient"):
        E = _log_int(rng, 4, 256)
        T = _log_int(rng, 1, 65536)
        return {"kind": kind, "T": T, "E": E, "k": min(E, rng.choice((1, 2, 4, 8))), "type": typ,
                "masked": rng.choice((0.0, 0.05)) if T >= 16 else 0.0}
    if kind == "orthogonalize":
        R, C = _log_int(rng, 16, 4096), _log_int(rng, 16, 4096)
        if rng.random() < 0.5:  # most sizes of real layers divide
            R, C = -(-R // 64) * 64, -(-C // 64) * 64
        B = min(rng.choice((1, 1, 4, 16)), max(1, (1 << 25) // (R * C)))
        return {"kind": kind, "B": B, "R": R, "C": C, "type": typ}
    if kind == "quantize":
        R, C = _log_int(rng, 32, 8192), _log_int(rng, 64, 8192)
        return {"kind": kind, "B": min(rng.choice((1, 8)), max(1, (1 << 26) // (R * C))), "R": R, "C": C, "type": typ}
    typ = rng.choice(("bf16", "f16"))
    out = rng.choice((typ, typ, "f32"))
    N, K = _log_int(rng, 128, 8192), _log_int(rng, 128, 8192)
    if rng.random() < 0.5:
        N, K = -(-N // 128) * 128, -(-K // 128) * 128
    if kind == "product":
        return {"kind": kind, "M": _log_int(rng, 1, 256), "N": N, "K": K, "type": typ, "out": out}
    E = _log_int(rng, 4, 64)
    N = min(N, 4096)
    K = min(K, 4096, max(128, (1 << 27) // (E * N)))
    T = _log_int(rng, 1, 256)
    return {"kind": kind, "T": T, "k": rng.choice((1, 2, 4)), "E": E, "N": N, "K": K, "type": typ, "out": out,
            "masked": rng.choice((0.0, 0.1)) if T >= 16 else 0.0}


# -- inputs -----------------------------------------------------------------------


def _values(shape, g):
    """Activations as layers see them: normal values, some columns much larger."""
    x = torch.randn(shape, generator=g, device="cuda")
    big = torch.rand(shape[-1], generator=g, device="cuda") < 0.01
    return x * torch.where(big, 20.0, 1.0)


def _logits(case, g):
    """A router's logits, some experts liked better; a masked token has none."""
    T, E = case["T"], case["E"]
    x = torch.randn((T, E), generator=g, device="cuda") + 0.5 * torch.randn(E, generator=g, device="cuda")
    gone = torch.rand(T, generator=g, device="cuda") < case["masked"]
    return torch.where(gone[:, None], torch.full_like(x, -math.inf), x).to(TYPES[case["type"]])


def _gradients(case, g):
    """Weight gradients: a few directions that stand out, over noise."""
    B, R, C = case["B"], case["R"], case["C"]
    r = max(1, min(R, C) // 16)
    size = torch.arange(1, r + 1, device="cuda").float().rsqrt()
    u, v = torch.randn((B, R, r), generator=g, device="cuda"), torch.randn((B, r, C), generator=g, device="cuda")
    x = torch.matmul(u * size, v) + 0.3 * torch.randn((B, R, C), generator=g, device="cuda")
    x = (1e-3 * x).to(TYPES[case["type"]])
    return x if B > 1 else x[0]


def _ids(case, g):
    """The k experts of each token, uneven over the experts; a masked token has none (-1)."""
    T, k, E = case["T"], case["k"], case["E"]
    score = torch.rand((T, E), generator=g, device="cuda").log().neg().log().neg()  # Gumbel
    score += torch.randn(E, generator=g, device="cuda")
    ids = score.topk(k, dim=1).indices.to(torch.int32)
    gone = torch.rand(T, generator=g, device="cuda") < case["masked"]
    return torch.where(gone[:, None], torch.full_like(ids, -1), ids).contiguous()


def _plain_sort(ids, E):
    """offsets of the experts and the token of each sorted row (-1 past the last)."""
    flat = ids.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < E), flat, torch.full_like(flat, E))
    order = key.sort(stable=True).indices
    offsets = torch.searchsorted(key[order], torch.arange(E + 1, device=ids.device), right=False).to(torch.int32)
    return offsets, torch.where(key[order] < E, order // ids.shape[1], -torch.ones_like(order)).to(torch.int32)


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, s = case["kind"], {"case": case}
    if kind == "choose":
        s["logits"] = _logits(case, g)
    elif kind == "choose_gradient":
        s["logits"] = _logits(case, g)
        s["weights"], s["ids"], s["counts"], _ = _plain_choose(s["logits"], case["k"])
        s["dweights"] = torch.randn((case["T"], case["k"]), generator=g, device="cuda") / case["T"]
        s["dloss"] = torch.rand((), generator=g, device="cuda") * 0.02 + 0.01
    elif kind == "orthogonalize":
        s["G"] = _gradients(case, g)
    elif kind == "quantize":
        shape = (case["R"], case["C"]) if case["B"] == 1 else (case["B"], case["R"], case["C"])
        s["w"] = (torch.randn(shape, generator=g, device="cuda") / math.sqrt(case["C"])).to(TYPES[case["type"]])
    else:
        N, K = case["N"], case["K"]
        if kind == "grouped":
            ids = _ids(case, g)
            s["offsets"], s["token"] = _plain_sort(ids, case["E"])
            s["most"] = max(1, int(s["offsets"].diff().max()))  # rows of the largest group
        rows, lead = (case["M"], ()) if kind == "product" else (case["T"], (case["E"],))
        s["x"] = _values((rows, K), g).to(TYPES[case["type"]])
        s["w"] = _plain_quantize((torch.randn(lead + (N, K), generator=g, device="cuda") / math.sqrt(K)))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own and case["kind"] in ("product", "grouped"):  # the library's object for the same weights
        from paper_2506_11209_amd import fp4
        s["W"] = fp4.quantize_weight(_plain_values(s.pop("w")))
    return s


# -- plain forms ------------------------------------------------------------------


def _plain_softmax(x):
    m = x.amax(-1, keepdim=True)
    e = (x - torch.where(m == -math.inf, torch.zeros_like(m), m)).exp()
    n = e.sum(-1, keepdim=True)
    return e / torch.where(n == 0, torch.ones_like(n), n)


def _plain_choose(logits, k):
    x = logits.float()
    T, E = x.shape
    p = _plain_softmax(x)
    top, at = x.sort(dim=1, descending=True, stable=True)
    top, at = top[:, :k], at[:, :k]
    there = top != -math.inf
    ids = torch.where(there, at, torch.full_like(at, -1)).to(torch.int32)
    weights = _plain_softmax(top)
    counts = torch.zeros(E + 1, dtype=torch.int32, device=x.device)
    counts.index_add_(0, torch.where(there, at, torch.full_like(at, E)).reshape(-1), there.reshape(-1).to(torch.int32))
    counts[E] = there[:, 0].sum()
    c, n = counts[:E].double(), counts[E].double()
    loss = E * (c * p.sum(0, dtype=torch.float64)).sum() / (c.sum() * n).clamp(min=1)
    return weights, ids, counts, loss.float()


def _plain_choose_gradient(s):
    x, w, dw = s["logits"].float(), s["weights"], s["dweights"]
    E = x.shape[1]
    p = _plain_softmax(x)
    c, n = s["counts"][:E].double(), s["counts"][E].double()
    scale = (E * s["dloss"].double() / (c.sum() * n).clamp(min=1)).float()
    c = c.float()
    d = scale * p * (c - (p * c).sum(1, keepdim=True))
    of_weights = w * (dw - (w * dw).sum(1, keepdim=True))
    there = s["ids"] >= 0
    d.scatter_add_(1, torch.where(there, s["ids"], torch.zeros_like(s["ids"])).long(), torch.where(there, of_weights, torch.zeros_like(w)))
    return d.to(s["logits"].dtype)


def _plain_orthogonalize(G):
    X = G.float()
    n = X.double().square().sum((-2, -1), keepdim=True).sqrt().float()
    X = X / torch.where(n == 0, torch.ones_like(n), n)
    tall = X.shape[-2] > X.shape[-1]
    if tall:
        X = X.transpose(-1, -2).contiguous()
    for _ in range(STEPS):
        A = torch.matmul(X, X.transpose(-1, -2).contiguous())
        X = A1 * X + torch.matmul(A3 * A + A5 * torch.matmul(A, A), X)
    return (X.transpose(-1, -2) if tall else X).bfloat16().contiguous()


def _plain_quantize(w):
    """(values of the codes, scales) of w (..., rows, columns), columns padded to blocks."""
    C = w.shape[-1]
    n = -(-C // BLOCK)
    v = torch.nn.functional.pad(w.float(), (0, n * BLOCK - C)).reshape(*w.shape[:-1], n, BLOCK)
    amax = v.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(amax)  # amax = m 2^e, 0.5 <= m < 1; 6 = 0.75 * 2^3
    e = torch.where(m <= 0.75, e - 3, e - 2)
    e = torch.where(amax > 0, e, torch.zeros_like(e)).clamp(-127, 127).to(torch.int32)
    y = torch.ldexp(v, -e)
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (a / step).round() * step  # ties to even codes
    return torch.where(y < 0, -a, a), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu).squeeze(-1), C


def _plain_values(q):
    codes, scales, C = q
    return (codes * scales.float()[..., None]).flatten(-2)[..., :C].contiguous()


def _plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "choose":
        return _plain_choose(s["logits"], case["k"])
    if kind == "choose_gradient":
        return _plain_choose_gradient(s)
    if kind == "orthogonalize":
        return _plain_orthogonalize(s["G"])
    if kind == "quantize":
        q = _plain_quantize(s["w"])
        return _plain_values(q).bfloat16(), q[1]
    w, x, out = _plain_values(s["w"]), s["x"].float(), TYPES[case["out"]]
    if kind == "product":
        return (x @ w.t()).to(out)
    offsets = s["offsets"]
    i = offsets[:-1, None] + torch.arange(s["most"], device=x.device)
    inside = i < offsets[1:, None]
    token = s["token"][torch.where(inside, i, torch.zeros_like(i))].clamp(min=0)
    c = torch.matmul(x[token], w.transpose(1, 2).contiguous())  # groups x most x columns
    r = torch.arange(s["token"].shape[0], device=x.device)
    g = torch.searchsorted(offsets[1:].long(), r, right=True)
    there, g = g < case["E"], g.clamp(max=case["E"] - 1)
    j = torch.where(there, r - offsets[g], torch.zeros_like(r))
    return torch.where(there[:, None], c[g, j], torch.zeros((), device=x.device)).to(out)


# -- one pass ---------------------------------------------------------------------


def _own(s):
    from paper_2506_11209_amd import experts, fp4, orthogonal
    case, kind = s["case"], s["case"]["kind"]
    if kind == "choose":
        return experts.choose(s["logits"], case["k"])
    if kind == "choose_gradient":
        return experts.choose_gradient(s["dweights"], s["dloss"], s["logits"], s["weights"], s["ids"], s["counts"])
    if kind == "orthogonalize":
        return orthogonal.orthogonalize(s["G"])
    if kind == "quantize":
        q = fp4.quantize_weight(s["w"])
        return q.dequantize("bf16"), q.scales
    if kind == "product":
        return fp4.product(s["x"], s["W"], out_dtype=case["out"])
    return fp4.grouped_product(s["x"], s["W"], s["offsets"], index=s["token"], out_dtype=case["out"])


def run(state):
    return _own(state) if own else _plain(state)


# -- what a pass cannot do without --------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind in ("choose", "choose_gradient"):
        T, E, k, size = case["T"], case["E"], case["k"], SIZE[case["type"]]
        if kind == "choose":
            return {"bytes": T * E * size + T * k * 8 + E * 4 + 8, "flops": 4 * T * E}
        return {"bytes": 2 * T * E * size + T * k * 12 + E * 4 + 8, "flops": 8 * T * E}
    if kind == "orthogonalize":
        B, R, C = case["B"], case["R"], case["C"]
        n, m = min(R, C), max(R, C)
        # half of each symmetric product, the whole of the third
        return {"bytes": B * R * C * (SIZE[case["type"]] + 2), "flops": STEPS * B * (3 * n * n * m + n * n * n)}
    if kind == "quantize":
        n = case["B"] * case["R"] * case["C"]
        return {"bytes": n * (SIZE[case["type"]] + 2) + n // 2 + n // BLOCK, "flops": 4 * n}
    N, K = case["N"], case["K"]
    weights = N * K // 2 + N * K // BLOCK
    if kind == "product":
        M = case["M"]
        return {"bytes": weights + M * K * 2 + M * N * SIZE[case["out"]], "flops": 2 * M * N * K}
    T, k, E = case["T"], case["k"], case["E"]
    R = T * k * (1 - case["masked"])
    used = E * (1 - (1 - 1 / E) ** R)  # experts that have rows
    return {"bytes": used * weights + T * K * 2 + T * k * N * SIZE[case["out"]], "flops": 2 * R * N * K}


# -- the definition in 64 bits --------------------------------------------------------


def _exact_softmax(x):
    e = torch.exp(x - x.max(1, keepdim=True).values)
    return torch.nan_to_num(e / e.sum(1, keepdim=True), nan=0.0)


def _exact_codes(w):
    """(values, scales) of rows x columns by the definition: the nearest of all codes."""
    R, C = w.shape
    n = -(-C // BLOCK)
    v = torch.zeros(R, n * BLOCK, dtype=torch.float64, device=w.device)
    v[:, :C] = w.double()
    v = v.view(R, n, BLOCK)
    amax = v.abs().max(-1).values
    scale = torch.ones_like(amax)
    some = amax > 0
    scale[some] = torch.exp2(torch.floor(torch.log2(amax[some] / 6.0)) - 1)  # one below at the most
    for _ in range(3):
        scale = torch.where(some & (amax > 6.0 * scale), 2 * scale, scale)
    y = v.abs() / scale[..., None]
    codes = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=w.device)
    between = (codes[1:] + codes[:-1]) / 2
    up = torch.bucketize(y.contiguous(), between)                # a value halfway stays below
    over = torch.bucketize(y.contiguous(), between, right=True)  # and here goes above
    at = torch.where((up != over) & (up % 2 == 1), over, up)
    return (codes[at] * torch.sign(v) * scale[..., None]).view(R, n * BLOCK)[:, :C], scale


def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind in ("choose", "choose_gradient"):
        x, E, k = s["logits"].double(), case["E"], case["k"]
        p = _exact_softmax(x)
        chosen = torch.zeros_like(x, dtype=torch.bool)
        left = x.clone()
        ids = []
        for _ in range(k):
            best = left.max(1, keepdim=True).values
            first = (left == best).to(torch.uint8).argmax(1, keepdim=True)  # the lowest of equals
            ids.append(first)
            chosen.scatter_(1, first, best > -math.inf)
            left.scatter_(1, first, -math.inf)
        ids = torch.cat(ids, 1)
        w = _exact_softmax(torch.gather(x, 1, ids))
        c = chosen.sum(0).double()
        n = chosen.any(1).sum().double()
        if kind == "choose":
            return w, None, None, E * (c / c.sum().clamp(min=1) * p.sum(0) / n.clamp(min=1)).sum()
        g = s["dloss"].double() * E * c / c.sum().clamp(min=1) / n.clamp(min=1)  # dloss / dp
        d = p * (g - (p * g).sum(1, keepdim=True))
        dw = s["dweights"].double()
        there = torch.gather(chosen, 1, ids)
        d.scatter_add_(1, ids, torch.where(there, w * (dw - (w * dw).sum(1, keepdim=True)), 0.0))
        return d
    if kind == "orthogonalize":
        G = s["G"].reshape(case["B"], case["R"], case["C"])
        out = torch.empty(G.shape, dtype=torch.float64, device="cuda")
        for i in range(case["B"]):
            X = G[i].double()
            X = X / X.norm()
            for _ in range(STEPS):  # from the shorter side
                if case["R"] <= case["C"]:
                    A = X @ X.t()
                    X = A1 * X + A3 * (A @ X) + A5 * (A @ (A @ X))
                else:
                    A = X.t() @ X
                    X = A1 * X + A3 * (X @ A) + A5 * ((X @ A) @ A)
            out[i] = X
        return out if case["B"] > 1 else out[0]
    if kind == "quantize":
        w = s["w"].reshape(-1, case["C"])
        parts = [_exact_codes(p) for p in w.split(16384)]
        shape = s["w"].shape[:-1]
        return torch.cat([p[0] for p in parts]).view(*shape, -1), torch.cat([p[1] for p in parts]).view(*shape, -1)
    codes, scales, K = s["w"]
    values = lambda c, e: (c.double() * e.double()[..., None]).flatten(-2)[:, :K]  # noqa: E731
    x = s["x"].double()
    if kind == "product":
        return x @ values(codes, scales).t()
    out = torch.zeros(s["token"].shape[0], case["N"], dtype=torch.float64, device="cuda")
    bounds, token = s["offsets"].tolist(), s["token"].long()
    for e in range(case["E"]):
        lo, hi = bounds[e], bounds[e + 1]
        if hi > lo:
            out[lo:hi] = x[token[lo:hi]] @ values(codes[e], scales[e]).t()
    return out
