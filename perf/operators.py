"""Operators of the 8-bit path: quantisation by blocks, the block-scaled product, its
grouped forms, and the routing of tokens to experts.

Each case is one pass through the public Python entry points (``own`` true:
``paper_2506_11209_amd.fp8`` and ``paper_2506_11209_amd.experts``) or through the
plain form of the same operator in elementary torch operations (``own`` false).

Formats: codes are e4m3 (OCP, largest value 448); a scale is a power of two in 8
bits (E8M0) for 128 values along the contraction, of one row or of 128 rows.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _up(n, m):
    return -(-n // m) * m


# -- cases ------------------------------------------------------------------------


def listed():
    return [
        # A decoding step's activations before a linear layer: latency.
        {"name": "quantize_rows_16x4096", "kind": "quantize", "form": "rows", "R": 16, "C": 4096, "type": "bf16"},
        # Activations of a training step: codes for the product and, transposed,
        # for the weight gradient, from one read.
        {"name": "quantize_both_8192x4096", "kind": "quantize", "form": "both", "R": 8192, "C": 4096, "type": "bf16"},
        # A master weight of ragged size after an optimizer step, in 128 x 128
        # blocks, with its transpose for the input gradient.
        {"name": "quantize_weight_4100x4104", "kind": "quantize", "form": "weight", "R": 4100, "C": 4104, "type": "f32"},
        # One token through a linear layer: the weight is read once.
        {"name": "product_1x8192x8192", "kind": "product", "form": "weight", "M": 1, "N": 8192, "K": 8192,
         "out": "bf16", "beta": 0.0},
        # The benchmark's cube as a forward product: the matrix rate.
        {"name": "product_8192x8192x8192", "kind": "product", "form": "weight", "M": 8192, "N": 8192, "K": 8192,
         "out": "bf16", "beta": 0.0},
        # A weight gradient that accumulates in 32 bits, of ragged sizes, both
        # operands with a scale for each row.
        {"name": "product_gradient_4104x1000x4100", "kind": "product", "form": "rows", "M": 4104, "N": 1000,
         "K": 4100, "out": "f32", "beta": 1.0},
        # A decoding batch of 32 tokens, four experts of 64 each: most experts
        # have a few rows, some none.
        {"name": "grouped_decode_32of64", "kind": "grouped", "T": 32, "k": 4, "E": 64, "N": 4096, "K": 2048,
         "out": "bf16", "masked": 0.0},
        # The same layer in training, unevenly loaded.
        {"name": "grouped_8192of16", "kind": "grouped", "T": 8192, "k": 2, "E": 16, "N": 4096, "K": 2048,
         "out": "bf16", "masked": 0.05},
        # Its weight gradient: contractions over as many rows as each expert has.
        {"name": "grouped_gradient_8192of16", "kind": "grouped_gradient", "T": 8192, "k": 2, "E": 16, "N": 1024,
         "K": 2048, "out": "f32", "masked": 0.05},
        # A training batch sorted by expert, its rows gathered.
        {"name": "route_8192x4of64", "kind": "route", "T": 8192, "k": 4, "E": 64, "C": 2048, "type": "bf16",
         "masked": 0.02},
        # A decoding batch's expert outputs back to its tokens.
        {"name": "combine_32x4of64", "kind": "combine", "T": 32, "k": 4, "E": 64, "C": 4096, "type": "bf16",
         "masked": 0.0},
        # The gradient of that step in training.
        {"name": "combine_gradient_8192x4of64", "kind": "combine_gradient", "T": 8192, "k": 4, "E": 64, "C": 2048,
         "type": "bf16", "masked": 0.02},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("quantize", "quantize", "product", "product", "product", "grouped", "grouped", "grouped_gradient",
                       "route", "combine", "combine_gradient"))
    typ = rng.choice(("bf16", "bf16", "f16", "f32"))
    if kind == "quantize":
        return {"kind": kind, "form": rng.choice(("rows", "both", "weight")), "R": _log_int(rng, 1, 8192),
                "C": _log_int(rng, 64, 8192), "type": typ}
    if kind == "product":
        c = {"kind": kind, "form": rng.choice(("weight", "weight", "rows")), "M": _log_int(rng, 1, 8192),
             "N": _log_int(rng, 128, 8192), "K": _log_int(rng, 128, 8192), "out": typ}
        if rng.random() < 0.5:  # most sizes of real layers divide
            c["N"], c["K"] = _up(c["N"], 128), _up(c["K"], 128)
        c["beta"] = 1.0 if c["form"] == "rows" else 0.0
        return c
    E = _log_int(rng, 4, 64)
    c = {"kind": kind, "T": _log_int(rng, 1, 8192), "k": rng.choice((1, 2, 4)), "E": E}
    c["masked"] = rng.choice((0.0, 0.0, 0.1)) if c["T"] >= 16 else 0.0
    if kind in ("grouped", "grouped_gradient"):
        most = 1 << 27  # elements of all experts' weights
        c["N"] = _log_int(rng, 128, 4096)
        c["K"] = min(_log_int(rng, 128, 4096), max(128, most // (E * c["N"])))
        if rng.random() < 0.5:
            c["N"], c["K"] = _up(c["N"], 128), _up(c["K"], 128)
        c["out"] = "f32" if kind == "grouped_gradient" else rng.choice(("bf16", "f16"))
    else:
        c["C"], c["type"] = _log_int(rng, 64, 4096), typ
    return c


# -- inputs -----------------------------------------------------------------------


def _values(shape, g, spread=1.0):
    """Activations as layers see them: normal values, some columns much larger."""
    x = torch.randn(shape, generator=g, device="cuda")
    big = torch.rand(shape[-1], generator=g, device="cuda") < 0.01
    return x * torch.where(big, 20.0 * spread, spread)


def _ids(case, g):
    """The k experts of each token, uneven over the experts; a masked token has none (-1)."""
    T, k, E = case["T"], case["k"], case["E"]
    score = torch.rand((T, E), generator=g, device="cuda").log().neg().log().neg()  # Gumbel
    score += torch.randn(E, generator=g, device="cuda")
    ids = score.topk(k, dim=1).indices.to(torch.int32)
    gone = torch.rand(T, generator=g, device="cuda") < case["masked"]
    return torch.where(gone[:, None], torch.full_like(ids, -1), ids).contiguous()


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, s = case["kind"], {"case": case}
    if kind == "quantize":
        s["x"] = _values((case["R"], case["C"]), g).to(TYPES[case["type"]])
    elif kind == "product":
        M, N, K = case["M"], case["N"], case["K"]
        s["A"] = _plain_rows(_values((M, K), g))
        w = torch.randn((N, K), generator=g, device="cuda") / math.sqrt(K)
        s["B"] = _plain_rows(w) if case["form"] == "rows" else _plain_weight(w)
        if case["beta"]:
            s["C0"] = torch.randn((M, N), generator=g, device="cuda").to(TYPES[case["out"]])
    elif kind in ("grouped", "grouped_gradient"):
        ids = _ids(case, g)
        s["offsets"], s["token"], s["place"] = _plain_sort(ids, case["E"])
        R, E, N, K = ids.numel(), case["E"], case["N"], case["K"]
        counts = s["offsets"].diff()
        s["most"] = max(1, int(counts.max()))  # rows of the largest group
        if kind == "grouped":
            s["A"] = _plain_rows(_values((R, K), g))
            w = torch.randn((E, N, K), generator=g, device="cuda") / math.sqrt(K)
            s["B"] = _plain_weight(w)
        else:
            s["A"] = _plain_columns(_values((R, N), g, 0.01), s["offsets"])
            s["B"] = _plain_columns(_values((R, K), g), s["offsets"])
    else:
        s["ids"] = _ids(case, g)
        R, T, C = s["ids"].numel(), case["T"], case["C"]
        if kind == "route":
            s["x"] = _values((T, C), g).to(TYPES[case["type"]])
        else:
            s["offsets"], s["token"], s["place"] = _plain_sort(s["ids"], case["E"])
            s["h"] = _values((R, C), g).to(TYPES[case["type"]])
            s["weights"] = torch.rand((T, case["k"]), generator=g, device="cuda").softmax(1)
            if kind == "combine_gradient":
                s["dy"] = _values((T, C), g, 0.01).to(TYPES[case["type"]])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:  # the library's objects for the same tensors
        from paper_2506_11209_amd import experts, fp8
        kind = case["kind"]
        rows = {"product": case.get("M"), "grouped": s["A"][0].shape[0] if "A" in s else 0, "grouped_gradient": case.get("N")}
        if kind in rows:
            deep = s["A"][0].shape[1] if kind == "grouped_gradient" else case["K"]
            s["A"] = fp8.Fp8Matrix(*s["A"], rows[kind], deep, 1)
            s["B"] = fp8.Fp8Matrix(*s["B"], case["K"] if kind == "grouped_gradient" else case["N"], deep,
                                   1 if kind == "grouped_gradient" or case.get("form") == "rows" else BLOCK)
        elif "place" in s:
            s["routes"] = experts.Routes(s["offsets"], s["token"], s["place"])
    return s


# -- plain forms ------------------------------------------------------------------


def _pad(x, rows, cols):
    return torch.nn.functional.pad(x, (0, cols - x.shape[-1], 0, rows - x.shape[-2])) if tuple(x.shape[-2:]) != (rows, cols) else x


def _plain_codes(x, amax):
    """Codes of x under blocks whose largest finite magnitude is amax (it
    broadcasts), and the scales' exponents plus 127."""
    m, e = torch.frexp(amax)  # amax = m 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    e = torch.where(amax > 0, e, torch.zeros_like(e)).clamp(-127, 127).to(torch.int32)
    by = ((127 - e) << 23).view(torch.float32)
    return torch.where(x.isfinite(), x * by, torch.full_like(x, math.nan)).to(E4M3), (e + 127).to(torch.uint8)


def _plain_rows(x):
    """(codes, scales) of x with a scale for 1 x 128 values."""
    R, C = x.shape
    n = -(-C // BLOCK)
    v = _pad(x.float(), R, n * BLOCK).reshape(R, n, BLOCK)
    amax = torch.where(v.isfinite(), v.abs(), torch.zeros_like(v)).amax(-1, keepdim=True)
    codes, e = _plain_codes(v, amax)
    return codes.reshape(R, n * BLOCK)[:, : _up(C, 16)].contiguous(), e.reshape(R, n).t().contiguous().view(E8M0)


def _plain_segments(offsets, R):
    """For each row of the padded order (each group starts at a multiple of 128)
    its source row, and whether it has one."""
    E = offsets.numel() - 1
    blocks = (R + (BLOCK - 1) * min(E, R)) // BLOCK
    counts = offsets.diff()
    ends = ((counts + BLOCK - 1) // BLOCK * BLOCK).cumsum(0)
    p = torch.arange(blocks * BLOCK, device=offsets.device)
    g = torch.searchsorted(ends, p, right=True)
    inside = g < E
    g = g.clamp(max=E - 1)
    starts = ends - (counts + BLOCK - 1) // BLOCK * BLOCK
    r = offsets[g] + p - starts[g]
    inside &= r < offsets[g + 1]
    return torch.where(inside, r, torch.zeros_like(r)), inside


def _plain_columns(x, offsets=None):
    """(codes, scales) of x transposed; with groups, in the padded order."""
    x = x.float()
    if offsets is not None:
        r, inside = _plain_segments(offsets, x.shape[0])
        x = torch.where(inside[:, None], x[r], torch.zeros((), device=x.device))
    return _plain_rows(x.t())


def _plain_weight(w):
    """(codes, scales) of w (..., N, K) with a scale for 128 x 128 values."""
    N, K = w.shape[-2:]
    a, b = -(-N // BLOCK), -(-K // BLOCK)
    v = _pad(w.float(), a * BLOCK, b * BLOCK).reshape(*w.shape[:-2], a, BLOCK, b, BLOCK)
    amax = torch.where(v.isfinite(), v.abs(), torch.zeros_like(v)).amax((-3, -1), keepdim=True)
    codes, e = _plain_codes(v, amax)
    codes = codes.reshape(*w.shape[:-2], a * BLOCK, b * BLOCK)[..., :N, : _up(K, 16)].contiguous()
    return codes, e.reshape(*w.shape[:-2], a, b).transpose(-1, -2).contiguous().view(E8M0)


def _plain_dequant(q, block_rows):
    codes, scales = q
    s = scales.float().transpose(-1, -2).repeat_interleave(BLOCK, -1)[..., : codes.shape[-1]]
    if block_rows > 1:
        s = s.repeat_interleave(block_rows, -2)[..., : codes.shape[-2], :]
    return codes.float() * s


def _plain_sort(ids, E):
    """offsets of the experts, the token of each sorted row (-1 past the last),
    the sorted row of each slot (-1: none); slots of an expert in their order."""
    flat = ids.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < E), flat, torch.full_like(flat, E))
    order = key.sort(stable=True).indices
    bounds = torch.arange(E + 1, device=ids.device)
    offsets = torch.searchsorted(key[order], bounds, right=False).to(torch.int32)
    place = torch.empty_like(flat)
    place[order] = torch.arange(flat.numel(), device=ids.device)
    token = torch.where(key[order] < E, order // ids.shape[1], -torch.ones_like(order)).to(torch.int32)
    place = torch.where(key < E, place, -torch.ones_like(place)).to(torch.int32).reshape(ids.shape)
    return offsets, token, place


def _plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "quantize":
        x = s["x"]
        if case["form"] == "rows":
            return _plain_rows(x)
        if case["form"] == "both":
            return _plain_rows(x), _plain_columns(x)
        return _plain_weight(x), _plain_weight(x.t())
    if kind == "product":
        r = _plain_dequant(s["A"], 1) @ _plain_dequant(s["B"], 1 if case["form"] == "rows" else BLOCK).t()
        return (r + case["beta"] * s["C0"].float() if case["beta"] else r).to(TYPES[case["out"]])
    if kind == "grouped":
        a, b, offsets = _plain_dequant(s["A"], 1), _plain_dequant(s["B"], BLOCK), s["offsets"]
        i = offsets[:-1, None] + torch.arange(s["most"], device=a.device)
        inside = i < offsets[1:, None]
        a = torch.where(inside[..., None], a[torch.where(inside, i, torch.zeros_like(i))], torch.zeros((), device=a.device))
        c = torch.matmul(a, b.transpose(1, 2))
        r = torch.arange(s["A"][0].shape[0], device=a.device)
        g = torch.searchsorted(offsets[1:].long(), r, right=True)
        inside, g = g < case["E"], g.clamp(max=case["E"] - 1)
        j = torch.where(inside, r - offsets[g], torch.zeros_like(r))
        return torch.where(inside[:, None], c[g, j], torch.zeros((), device=a.device)).to(TYPES[case["out"]])
    if kind == "grouped_gradient":
        a, b = _plain_dequant(s["A"], 1), _plain_dequant(s["B"], 1)
        n = (s["offsets"].diff() + BLOCK - 1) // BLOCK * BLOCK
        ends = n.cumsum(0)
        i = (ends - n)[:, None] + torch.arange(_up(s["most"], BLOCK), device=a.device)
        inside = i < ends[:, None]
        i = torch.where(inside, i, torch.zeros_like(i))
        a = a.t()[i] * inside[..., None]
        b = b.t()[i]
        return torch.matmul(a.transpose(1, 2), b)
    if kind == "route":
        offsets, token, place = _plain_sort(s["ids"], case["E"])
        x = s["x"]
        xs = torch.where((token >= 0)[:, None], x[token.clamp(min=0)], torch.zeros((), device=x.device, dtype=x.dtype))
        return offsets, token, place, xs
    place, w, h = s["place"].long(), s["weights"], s["h"]
    there = place >= 0
    hs = h[place.clamp(min=0)].float()  # T x k x C
    if kind == "combine":
        return (torch.where(there, w, torch.zeros_like(w))[..., None] * hs).sum(1).to(h.dtype)
    dy = s["dy"].float()
    dw = torch.where(there, (hs * dy[:, None]).sum(-1), torch.zeros_like(w))
    t = s["token"].clamp(min=0).long()
    row_w = torch.zeros(h.shape[0] + 1, device=h.device)
    row_w[torch.where(there, place, torch.full_like(place, h.shape[0]))] = w
    dh = torch.where((s["token"] >= 0)[:, None], dy[t] * row_w[:-1, None], torch.zeros((), device=h.device))
    return dh.to(h.dtype), dw


# -- one pass ---------------------------------------------------------------------


def _whole(q):
    return q.codes, q.scales


def _own(s):
    from paper_2506_11209_amd import experts, fp8
    case, kind = s["case"], s["case"]["kind"]
    if kind == "quantize":
        if case["form"] == "rows":
            return _whole(fp8.quantize_rows(s["x"]))
        return tuple(map(_whole, fp8.quantize_both(s["x"]) if case["form"] == "both" else fp8.quantize_weight(s["x"])))
    if kind == "product":
        return fp8.product(s["A"], s["B"], out_dtype=case["out"], beta=case["beta"], C0=s.get("C0"))
    if kind == "grouped":
        return fp8.grouped_product(s["A"], s["B"], s["offsets"], out_dtype=case["out"])
    if kind == "grouped_gradient":
        return fp8.grouped_gradient(s["A"], s["B"], s["token"].shape[0], s["offsets"], out_dtype=case["out"])
    if kind == "route":
        routes = experts.sort(s["ids"], case["E"])
        return routes.offsets, routes.token, routes.place, experts.gather(s["x"], routes)
    if kind == "combine":
        return experts.combine(s["h"], s["routes"], s["weights"])
    return experts.combine_gradient(s["dy"], s["h"], s["routes"], s["weights"])


def run(state):
    return _own(state) if own else _plain(state)


# -- what a pass cannot do without --------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind == "quantize":
        n = case["R"] * case["C"]
        codes = n if case["form"] == "rows" else 2 * n
        scales = codes // (BLOCK * BLOCK if case["form"] == "weight" else BLOCK)
        return {"bytes": n * SIZE[case["type"]] + codes + scales, "flops": 2 * n}
    if kind == "product":
        M, N, K = case["M"], case["N"], case["K"]
        scales = K // BLOCK * (M + (N if case["form"] == "rows" else N // BLOCK))
        return {"bytes": M * K + N * K + scales + (2 if case["beta"] else 1) * M * N * SIZE[case["out"]], "flops": 2 * M * N * K}
    T, k, E = case["T"], case["k"], case["E"]
    R = T * k * (1 - case["masked"])
    if kind in ("grouped", "grouped_gradient"):
        N, K = case["N"], case["K"]
        if kind == "grouped":
            used = E * (1 - (1 - 1 / E) ** R)  # experts that have rows
            return {"bytes": R * K + used * N * K + T * k * N * SIZE[case["out"]], "flops": 2 * R * N * K}
        return {"bytes": R * (N + K) + E * N * K * SIZE[case["out"]], "flops": 2 * R * N * K}
    C, size = case["C"], SIZE[case["type"]]
    if kind == "route":
        return {"bytes": T * k * 12 + (T + T * k) * C * size, "flops": 0}
    if kind == "combine":
        return {"bytes": T * k * 8 + (R + T) * C * size, "flops": 2 * R * C}
    return {"bytes": T * k * 12 + (2 * R + T) * C * size, "flops": 3 * R * C}


# -- the definition in 64 bits --------------------------------------------------------


def _two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_quant(x, br, bc):
    """(codes' values, scales) of x in blocks of br x bc, by the definition."""
    R, C = x.shape
    a, b = -(-R // br), -(-C // bc)
    v = torch.zeros(a * br, b * bc, dtype=torch.float64, device=x.device)
    v[:R, :C] = x.double()
    amax = v.view(a, br, b, bc).abs().permute(0, 2, 1, 3).reshape(a, b, br * bc).max(-1).values
    e = torch.zeros_like(amax)
    some = amax > 0
    e[some] = torch.floor(torch.log2(amax[some] / 448.0)) - 1  # one below at the most
    for _ in range(3):
        e = torch.where(some & (amax > 448.0 * _two_to(e)), e + 1, e)
    scale = _two_to(e)
    y = v / scale.repeat_interleave(br, 0).repeat_interleave(bc, 1)
    size = torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent - 1
    step = _two_to(size - 3)  # e4m3: three bits after the leading one, subnormals below 2^-6
    return (torch.round(y / step) * step)[:R, : _up(C, 16)], scale.t()


def _exact_matrix(q, row_block):
    c, s = q[0].double(), q[1].double()
    k = torch.arange(c.shape[-1], device=c.device) // BLOCK
    n = torch.arange(c.shape[-2], device=c.device) // row_block
    return c * s[..., k, :][..., n].transpose(-1, -2)


def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind == "quantize":
        x = s["x"]
        if case["form"] == "rows":
            return _exact_quant(x, 1, BLOCK)
        br = 1 if case["form"] == "both" else BLOCK
        return _exact_quant(x, br, BLOCK), _exact_quant(x.t(), br, BLOCK)
    if kind == "product":
        r = torch.mm(_exact_matrix(s["A"], 1), _exact_matrix(s["B"], 1 if case["form"] == "rows" else BLOCK).t().contiguous())
        return torch.add(r, s["C0"].double(), alpha=case["beta"]) if case["beta"] else r
    bounds = s["offsets"].tolist() if "offsets" in s else None
    if kind == "grouped":
        out = torch.zeros(s["A"][0].shape[0], case["N"], dtype=torch.float64, device="cuda")
        for g in range(case["E"]):
            lo, hi = bounds[g], bounds[g + 1]
            if hi > lo:
                a = _exact_matrix((s["A"][0][lo:hi], s["A"][1].view(torch.uint8)[:, lo:hi].contiguous().view(E8M0)), 1)
                out[lo:hi] = torch.mm(a, _exact_matrix((s["B"][0][g], s["B"][1][g]), BLOCK).t().contiguous())
        return out
    if kind == "grouped_gradient":
        out = torch.zeros(case["E"], case["N"], case["K"], dtype=torch.float64, device="cuda")
        a, b, at = _exact_matrix(s["A"], 1), _exact_matrix(s["B"], 1), 0
        for g in range(case["E"]):
            n = _up(bounds[g + 1] - bounds[g], BLOCK)
            if n:
                out[g] = torch.mm(a[:, at:at + n].contiguous(), b[:, at:at + n].t().contiguous())
            at += n
        return out
    if kind == "route":
        ids = s["ids"].cpu().reshape(-1).tolist()
        rows = sorted((e, i) for i, e in enumerate(ids) if 0 <= e < case["E"])
        x = s["x"].double()
        xs = torch.zeros(len(ids), case["C"], dtype=torch.float64, device="cuda")
        if rows:
            xs[: len(rows)] = x[torch.tensor([i // case["k"] for _, i in rows], device="cuda")]
        return None, None, None, xs
    place, w, h = s["place"].cpu(), s["weights"].double(), s["h"].double()
    T, k = place.shape
    dy = s["dy"].double() if "dy" in s else None
    y = torch.zeros(T, case["C"], dtype=torch.float64, device="cuda")
    dh, dw = torch.zeros_like(h), torch.zeros(T, k, dtype=torch.float64, device="cuda")
    for j in range(k):
        t = (place[:, j] >= 0).nonzero().flatten().cuda()
        p = place[:, j].cuda()[t].long()
        if dy is None:
            y[t] += w[t, j, None] * h[p]
        else:
            dh[p] = w[t, j, None] * dy[t]
            dw[t, j] = (dy[t] * h[p]).sum(1)
    return y if dy is None else (dh, dw)
