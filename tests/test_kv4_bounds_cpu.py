"""The oracle's bound of the 4-bit cache's attention, on the CPU: it holds for
what it allows and not for planted mistakes."""

import numpy as np
import pytest
import torch

from oracle import kv4 as O


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def case(d, rows=6, keys=80, std=1.3, seed=0):
    rng = np.random.default_rng(seed)
    K, V = (O.quantise(rng.normal(size=(keys, 2, d)) * std, g) for g in (32, d))
    q = bf16(rng.normal(size=(rows, 8, d)) * std)
    visible = np.tril(np.ones((rows, keys), bool), keys - rows)
    return q, K, V, visible


def test_e4m3():
    x = torch.tensor(np.random.default_rng(0).normal(size=4000) * 40.0)
    x = torch.cat([x, x * 2.0 ** -12, torch.tensor([0.0, 2.0 ** -10, 3 * 2.0 ** -10, 240.0, 247.9])])
    want = x.float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.e4m3(x.float().double().numpy()), want)


@pytest.mark.parametrize("d", [64, 128])
def test_query_loss(d):
    """Nothing in numbers less than 2^9 below the largest, 2^-17 of the largest at most in the others;
    with outliers 2^-34, however many of them."""
    q = bf16(np.random.default_rng(d).normal(size=(500, d)))
    top, lost = np.abs(q).max(-1, keepdims=True), O.query_loss(q)
    assert (lost[np.abs(q) >= top * 2.0 ** -9] == 0).all() and (lost <= 2.0 ** -17 * top).all()
    assert (lost <= np.abs(q)).all() and lost.any()
    for n in (1, 2, d // 2, d - 4):
        x = q.copy()
        x[:, :n] = 5000
        assert (O.query_loss(x) <= 2.0 ** -34 * 5000).all()


@pytest.mark.parametrize("d", [64, 128])
def test_bound_of_two_part_queries(d):
    """Two e4m3 parts alone in rows with two or four equal outliers are past the bound."""
    q, K, V, visible = case(d)
    dims = [5, 37] if d == 64 else [5, 37, 69, 101]
    K[:, :, dims] = 0
    q[:, :, dims] = 20000
    s = 2.0 ** (np.floor(np.log2(20000)) - 7)
    two = O.e4m3(q / s)
    two = (two + O.e4m3(q / s - two)) * s
    o, spread = O.attend(q, K, V, visible)
    tol = O.attend_bound(q, K, V, visible, o, spread)
    assert not (np.abs(O.attend(two, K, V, visible)[0] - o) <= tol).all()
    assert (np.abs(bf16(o) - o) <= tol).all()


def test_negative_zeros_are_counted():
    """A code 8 in either half of any code byte of K or V; scales that hold an 8 are none."""
    d, size = 64, 64 * (64 + 2 + 2)
    page = np.full(2 * 3 * size, 0xFF, np.uint8)
    heads = page.reshape(6, size)
    heads[:, 64 * d:] = 8
    assert O.negative_zeros(page, 2, 3, d) == 0
    heads[4, 7] = 0x81
    heads[5, 64 * d - 1] = 0x18
    assert O.negative_zeros(page, 2, 3, d) == 2


def test_bound_at_large_scores():
    """Scores of several hundred, off by 0.02 here and there: past the bound, which the exact output
    rounded to bf16 is not."""
    q, K, V, visible = case(128, rows=8, keys=508, std=8.0, seed=11)
    o, spread = O.attend(q, K, V, visible)
    tol = O.attend_bound(q, K, V, visible, o, spread)
    assert (np.abs(bf16(o) - o) <= tol).all()
    rng = np.random.default_rng(0)
    worst = 0.0
    for i in range(8):
        z = np.where(visible, q[:, i] @ K[:, i // 4].T / np.sqrt(128), -np.inf)
        z += 0.02 * rng.choice([-1.0, 1.0], size=z.shape)
        p = np.exp(z - z.max(1, keepdims=True))
        off = (p / p.sum(1, keepdims=True)) @ V[:, i // 4]
        worst = max(worst, (np.abs(off - o[:, i]) / tol[:, i]).max())
    assert worst > 1
