"""The router's choice, its loss and its gradient by their definitions, in 64 bits on
the CPU."""
import numpy as np


def softmax(x):
    """Over the last axis; zeros where all is -inf, NaN where a value is NaN or +inf."""
    with np.errstate(invalid="ignore"):
        m = x.max(-1, keepdims=True)
        e = np.exp(x - np.where(m == -np.inf, 0.0, m))
        n = e.sum(-1, keepdims=True)
        return e / np.where(n == 0, 1.0, n)


def choose(logits, k):
    """(weights, ids, counts, loss, p) of float64 logits."""
    x = np.asarray(logits, dtype=np.float64)
    T, E = x.shape
    order = np.where(np.isnan(x), np.inf, x) + 0.0
    nan = np.isnan(x)
    ids = np.full((T, k), -1, np.int32)
    for t in range(T):
        # NaN before all, then larger first, the lowest index first among equals
        rank = sorted(range(E), key=lambda e: (not nan[t, e], -order[t, e], e))
        chosen = [e for e in rank[:k] if nan[t, e] or x[t, e] != -np.inf]
        ids[t, : len(chosen)] = chosen
    there = ids >= 0
    top = np.where(there, np.take_along_axis(x, np.maximum(ids, 0).astype(np.int64), 1), -np.inf)
    w = np.where(there, softmax(top), 0.0)
    c = np.bincount(ids[there], minlength=E).astype(np.int64)
    n = int(there.any(1).sum())
    p = softmax(x)
    loss = E * (c * p.sum(0)).sum() / (c.sum() * n) if n else 0.0
    return w, ids, np.append(c, n).astype(np.int64), loss, p


def gradient(dweights, dloss, logits, k):
    x = np.asarray(logits, dtype=np.float64)
    w, ids, counts, _, p = choose(x, k)
    E = x.shape[1]
    c, n = counts[:E].astype(np.float64), counts[E]
    d = np.zeros_like(x)
    if n and dloss is not None:
        d += float(dloss) * E / (c.sum() * n) * p * (c - (p * c).sum(1, keepdims=True))
    if dweights is not None:
        of = w * (dweights - (w * dweights).sum(1, keepdims=True))
        for t in range(x.shape[0]):
            for j in range(k):
                if ids[t, j] >= 0:
                    d[t, ids[t, j]] += of[t, j]
    return d
