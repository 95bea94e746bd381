"""Oracle for the KV cache in 4 bits: what the cache stands for, its bytes, and
the attention over it.

TEST INFRASTRUCTURE ONLY.  Plain float64 numpy, written from the format's
definition; it shares no code with the product path.

A number is an E2M1 code times its group's power of two 2^e: 32 consecutive
numbers of a key make a group, so do all numbers of a value.  e is the smallest
exponent in [-126, 125] with max |x| <= 6 * 2^e, or 125; the code is the nearest
to x / 2^e, the even one of two equally near.  A group with an infinity or NaN
reads as NaN.
"""

import numpy as np

PAGE = 64
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def exponent(top):
    """The exponent of a group whose largest magnitude is ``top`` (finite)."""
    e = -126
    while top > 6.0 * 2.0 ** e and e < 125:
        e += 1
    return e


def quantise(x, group):
    """What the cache holds for x [..., n], groups of ``group`` numbers."""
    x = np.asarray(x, dtype=np.float64)
    flat = x.reshape(-1, group)
    out = np.empty_like(flat)
    for i, row in enumerate(flat):
        if not np.isfinite(row).all():
            out[i] = np.nan
            continue
        s = 2.0 ** exponent(np.abs(row).max())
        dist = np.abs(np.abs(row)[:, None] / s - GRID)
        near = dist == dist.min(axis=1, keepdims=True)
        even = near & (np.arange(8) % 2 == 0)
        code = np.where(even.any(axis=1), even.argmax(axis=1), near.argmax(axis=1))
        out[i] = np.sign(row) * GRID[code] * s
    return out.reshape(x.shape)


def rotate(k, pos, theta):
    """Half-split rotation of k [rows, heads, d] by positions pos [rows]."""
    k = np.asarray(k, dtype=np.float64)
    d = k.shape[-1]
    ang = np.asarray(pos, np.float64)[:, None, None] * theta ** (-2.0 * np.arange(d // 2) / d)
    a, b = k[..., :d // 2], k[..., d // 2:]
    return np.concatenate([a * np.cos(ang) - b * np.sin(ang), b * np.cos(ang) + a * np.sin(ang)], -1)


def stored(k, v, pos=None, theta=None):
    """What the cache holds for rows k, v [rows, heads, d]; pos: rotate k first."""
    with np.errstate(invalid="ignore"):
        if pos is not None:
            k = rotate(k, pos, theta)
        return quantise(k, 32), quantise(v, v.shape[-1])


def decode_page(page, n_layers, n_kv_heads, d):
    """A page's bytes -> K, V [layers, kv heads, 64, d], number by number of the layout."""
    K = np.empty((n_layers, n_kv_heads, PAGE, d))
    V = np.empty_like(K)
    size = PAGE * (d + d // 32 + 2)
    signed = np.concatenate([GRID, -GRID])
    for l in range(n_layers):
        for g in range(n_kv_heads):
            x = page[(l * n_kv_heads + g) * size:][:size]
            codes, scales = x[:PAGE * d], x[PAGE * d:]
            w = scales[PAGE * (d // 32):].view(np.uint16).astype(np.uint32) << 16
            vs = w.view(np.float32).astype(np.float64)
            for t in range(PAGE):
                for j in range(d):
                    at = t // 32 * (16 * d) + j // 32 * 512 + t % 32 * 16 + j % 32 // 2
                    e = int(scales[t * (d // 32) + j // 32])
                    s = np.nan if e == 255 else 2.0 ** (e - 127)
                    K[l, g, t, j] = signed[codes[at] >> 4 * (j % 2) & 15] * s
                    at = PAGE * d // 2 + t // 8 * (4 * d) + (j % 32 * (d // 32) + j // 32) * 4 + t % 8 // 2
                    V[l, g, t, j] = signed[codes[at] >> 4 * (t % 2) & 15] * vs[t]
    return K, V


def negative_zeros(page, n_layers, n_kv_heads, d):
    """How many numbers of a page's bytes have the code 8, which nothing is stored as."""
    heads = page[:n_layers * n_kv_heads * PAGE * (d + d // 32 + 2)].reshape(n_layers * n_kv_heads, -1)
    codes = heads[:, :PAGE * d]
    return int((codes & 15 == 8).sum() + (codes >> 4 == 8).sum())


def sees(parents, rows):
    """[rows, rows] whether row i sees row j, and the rows' depths; parents None: a run."""
    if parents is None:
        return np.tril(np.ones((rows, rows), bool)), np.arange(rows)
    m, depth = np.eye(rows, dtype=bool), np.zeros(rows, int)
    for i in range(1, rows):
        m[i] |= m[parents[i]]
        depth[i] = depth[parents[i]] + 1
    return m, depth


def attend(q, K, V, visible):
    """q [rows, heads, d], K, V [keys, kv heads, d], visible [rows, keys] -> (out, spread):
    out [rows, heads, d], and the same sum over |V| instead of V (what roundings of the
    probabilities scale with)."""
    rows, heads, d = q.shape
    group = heads // K.shape[1]
    out, spread = np.empty(q.shape), np.empty(q.shape)
    for i in range(heads):
        k, v = K[:, i // group], V[:, i // group]
        z = np.where(visible, q[:, i] @ np.where(np.isnan(k), np.nan, k).T / np.sqrt(d), -np.inf)
        p = np.exp(z - z.max(axis=1, keepdims=True))
        p /= p.sum(axis=1, keepdims=True)
        out[:, i], spread[:, i] = p @ v, p @ np.abs(v)
    return out, spread


def e4m3(x):
    """x rounded to e4m3 (4 significant bits, steps of 2^-9 at least), |x| < 448."""
    x = np.asarray(x, np.float64)
    e = np.maximum(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -20))), -6)
    return np.round(x * 2.0 ** (3 - e)) * 2.0 ** (e - 3)


def query_loss(q):
    """What each number of bf16 queries q [..., d] may be off by where the attention holds it as
    two e4m3 numbers of the row's power of two, or, in rows that lose more than 2^-12 of the
    numbers below a sixteenth of their largest, as four."""
    q = np.asarray(q, np.float64)
    top = np.abs(q).max(-1, keepdims=True)
    s = 2.0 ** np.maximum(np.floor(np.log2(np.maximum(top, 2.0 ** -140))) - 7, -126)
    rest = q / s
    for _ in range(2):
        rest = rest - e4m3(rest)
    lost = np.abs(rest) * s
    small = np.where(np.abs(q) < top / 16, np.abs(q), 0.0)
    wide = lost.sum(-1, keepdims=True) > 2.0 ** -12 * small.sum(-1, keepdims=True)
    return np.where(wide, np.minimum(lost, 2.0 ** -34 * top), lost)


def attend_bound(q, K, V, visible, out, spread):
    """How far the attention's output (rounded to bf16) may be from out = attend()[0], element by
    element, by its roundings; spread = attend()[1], arguments as there.

    Per row and head, with v = 2^-24 (fp32, half a step, relative): the score of a key is a sum of d
    products, off by at most (d + 2) v B, B = sum |q k| / sqrt(d) of that key; the scale and the
    subtraction of the reference add 4 v B, exp2 4 v; the query's parts what query_loss() says times
    |k| / sqrt(d).  The largest of it over the visible keys is e: the probabilities of a row change
    by factors within exp(+-2 e) against each other, the output by expm1(2 e) spread.  Rounding the
    probabilities to bf16 adds 2^-8 spread, sums over n keys and merges 2 (n + 70) v spread, numbers
    flushed below 2^-126 (n + 1) 2^-126 (max |V| + 6), and rounding the output 2^-8 of it."""
    rows, heads, d = q.shape
    group = heads // K.shape[1]
    bound = np.empty(out.shape)
    v, aq, lost = 2.0 ** -24, np.abs(q), query_loss(q)
    n = visible.sum(1)[:, None]
    for i in range(heads):
        k = np.abs(K[:, i // group]).T / np.sqrt(d)
        e = np.where(visible, (d + 6) * v * (aq[:, i] @ k) + lost[:, i] @ k, 0.0).max(1) + 4 * v
        bound[:, i] = (np.expm1(2 * e)[:, None] + 2.0 ** -8 + 2 * (n + 70) * v) * spread[:, i]
        bound[:, i] += (n + 1) * 2.0 ** -126 * (np.abs(V[:, i // group]).max() + 6)
    return bound + 2.0 ** -8 * (np.abs(out) + bound)
