"""Oracle for the operators of a drafting loop: products with weights in 4 bits,
the choice of beams, and the cache rows that follow them.

TEST INFRASTRUCTURE ONLY.  Plain float64 numpy, written from the definitions; it
shares no code with the product path.

A weight is an E2M1 code times a power of two 2^e that 32 consecutive numbers of a
row share: the smallest e in [-120, 125] with max |x| <= 6 * 2^e, or 125; the
nearest code, the even one of two equally near.  A group with an infinity or NaN
reads as NaN.
"""

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GROUP = 32


def quantise(w):
    """What a matrix [rows, cols] in 4 bits stands for."""
    w = np.asarray(w, dtype=np.float64)
    flat = w.reshape(-1, GROUP)
    out = np.empty_like(flat)
    for i, row in enumerate(flat):
        if not np.isfinite(row).all():
            out[i] = np.nan
            continue
        e, top = -120, np.abs(row).max()
        while top > 6.0 * 2.0 ** e and e < 125:
            e += 1
        s = 2.0 ** e
        dist = np.abs(np.abs(row)[:, None] / s - GRID)
        near = dist == dist.min(axis=1, keepdims=True)
        even = near & (np.arange(8) % 2 == 0)
        code = np.where(even.any(axis=1), even.argmax(axis=1), near.argmax(axis=1))
        out[i] = np.sign(row) * GRID[code] * s
    return out.reshape(w.shape)


def linear(x, w):
    """x W^T and sum |x w| of every output."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    return x @ w.T, np.abs(x) @ np.abs(w).T


def silu(g):
    with np.errstate(over="ignore"):
        return g / (1.0 + np.exp(-g))


def select(logits, scores, k, last=None, eos=-1):
    """(parents, tokens, scores) [groups, k] of the k best candidates of logits [groups, width,
    vocab]; -1, -1 and -inf where there are fewer."""
    z, s = np.asarray(logits, np.float64), np.asarray(scores, np.float64)
    groups, width, vocab = z.shape
    parents = np.full((groups, k), -1, np.int64)
    tokens = parents.copy()
    best = np.full((groups, k), -np.inf)
    for g in range(groups):
        key = np.full((width, vocab), -np.inf)
        for w in range(width):
            row = z[g, w]
            if not np.isfinite(s[g, w]):
                continue
            if eos >= 0 and last[g][w] == eos:
                key[w, eos] = s[g, w]
            elif not (np.isnan(row) | (row == np.inf)).any() and (row > -np.inf).any():
                top = row.max()
                key[w] = s[g, w] + (row - (top + np.log(np.exp(row - top).sum())))
        flat = key.ravel()
        order = np.lexsort((np.arange(flat.size), -flat))[:k]
        order = order[flat[order] > -np.inf]
        parents[g, :len(order)], tokens[g, :len(order)] = order // vocab, order % vocab
        best[g, :len(order)] = flat[order]
    return parents, tokens, best


def reorder(held, parents):
    """held: [groups][width] arrays of the beams' ranges; what they are afterwards."""
    out = []
    for beams, row in zip(held, parents):
        out.append([beams[p] if 0 <= p < len(beams) else beams[j] for j, p in enumerate(row)])
    return out
