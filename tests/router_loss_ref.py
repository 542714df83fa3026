"""Balance loss, z-loss, counts and logit gradients of the router in 64 bits,
token by token (numpy; the tests' reference)."""
import numpy as np


def softmax_row(y):
    """(p, lse) of one row; a row of -inf only has p = 0 and lse = 0."""
    m = y.max()
    if m == -np.inf:
        return np.zeros_like(y), 0.0
    e = np.exp(y - m)
    return e / e.sum(), m + np.log(e.sum())


def forward(logits, idx, off=None, mask=None):
    """(balance [G], zloss [G], counts [G][E], prob_sum [G][E], n [G])."""
    T, E = logits.shape
    k = idx.shape[1]
    off = [0, T] if off is None else list(off)
    G = len(off) - 1
    counts, psum = np.zeros((G, E), dtype=np.int64), np.zeros((G, E))
    z, n = np.zeros(G), np.zeros(G, dtype=np.int64)
    for g in range(G):
        for t in range(off[g], off[g + 1]):
            if mask is not None and not mask[t]:
                continue
            p, lse = softmax_row(logits[t].astype(np.float64))
            psum[g] += p
            z[g] += lse * lse
            n[g] += 1
            for e in idx[t]:
                if 0 <= e < E:
                    counts[g, e] += 1
    m = np.maximum(n, 1)
    return E / (k * m.astype(np.float64) ** 2) * (counts * psum).sum(1), z / m, counts, psum, n


def backward(logits, counts, n, db, dz, k, off=None, mask=None):
    T, E = logits.shape
    off = [0, T] if off is None else list(off)
    out = np.zeros((T, E))
    for g in range(len(off) - 1):
        if n[g] == 0:
            continue
        a = E * counts[g] / (k * float(n[g]))
        for t in range(off[g], off[g + 1]):
            if mask is not None and not mask[t]:
                continue
            p, lse = softmax_row(logits[t].astype(np.float64))
            out[t] = p * (db[g] / n[g] * (a - (a * p).sum()) + 2 * dz[g] / n[g] * lse)
    return out
