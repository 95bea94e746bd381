"""GPU parity of the 4-bit cache's attention against the float64 oracle within
oracle.kv4.attend_bound: element by element, every term from the row and the
keys that it sees."""

import numpy as np
import pytest
import torch

import paper_2512_04752_amd as sv
from oracle import kv4 as O
from tests.test_gpu_kv4 import Cache, bf16, config, random_tree

pytestmark = pytest.mark.gpu


def read(step, layer, n, kv, d):
    ko, vo = (torch.empty(n, kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sv.spec_kv4_read(step, layer, ko, vo)
    return tuple(t.double().cpu().numpy() for t in (ko, vo))


def check(q, out, K, V, visible, what):
    o, spread = O.attend(q, K, V, visible)
    err, tol = np.abs(out - o), O.attend_bound(q, K, V, visible, o, spread)
    assert (err <= tol).all(), f"{what}: error {err.max():.3g}, {(err / tol).max():.2f} of its bound"


@pytest.mark.parametrize("d,dims", [(64, (5, 37)), (64, tuple(range(0, 64, 2))), (64, tuple(range(60))),
                                    (128, (5, 69)), (128, (5, 37, 69, 101)), (128, tuple(range(1, 128, 2)))],
                         ids=lambda x: str(x if isinstance(x, int) else len(x)))
@pytest.mark.parametrize("ratio", [100.0, 1000.0, 5000.0, 20000.0, 2.0 ** 20])
def test_queries_with_several_outliers(d, dims, ratio):
    """Rows whose outliers, several of one size, lie where the keys are zero: the scores are those of the
    other numbers.  Ordinary rows between them come out as they do alone."""
    rows, dims = 24, list(dims)
    cfg = config(8, 2, d)
    rng = np.random.default_rng(len(dims) + int(ratio))
    c = Cache(cfg, [0], [rows])
    k = rng.normal(size=(rows, 2, d)) * 2
    k[:, :, dims] = 0
    step = c.append(0, [0], [0], bf16(k).cuda(), bf16(rng.normal(size=(rows, 2, d))).cuda(), [rows], rotate=False)
    K, V = read(step, 0, rows, 2, d)
    assert (K[:, :, dims] == 0).all()
    plain = rng.normal(size=(rows, 8, d))
    q = plain.copy()
    q[::2, :, dims] = ratio * rng.choice([-1.0, 1.0], size=q[::2, :, dims].shape)
    out, alone = (torch.empty(rows, 8 * d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sv.spec_kv4_attend(step, 0, bf16(q).cuda(), out)
    sv.spec_kv4_attend(step, 0, bf16(plain).cuda(), alone)
    assert torch.equal(out[1::2], alone[1::2])
    check(bf16(q).double().numpy(), out.double().cpu().numpy().reshape(q.shape), K, V,
          np.tril(np.ones((rows, rows), bool)), f"d {d}, {len(dims)} outliers of {ratio}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rotate", [True, False])
def test_no_negative_zero_is_stored(d, rotate):
    """Negative numbers too small for their group's steps, and -0: code 0, in every page and head, and
    read back as +0, in K and V."""
    rows, kv = 90, 256 // d
    cfg = config(kv, kv, d, layers=2)
    rng = np.random.default_rng(d)
    x = rng.normal(size=(2, rows, kv, d))
    x[rng.random(x.shape) < 0.5] *= 1e-3
    x[rng.random(x.shape) < 0.1] = -0.0
    x[:, 5] = -0.0
    x = bf16(x).cuda()
    c = Cache(cfg, [3], [rows])
    step = c.append(1, [0], [3], x[0], x[1], [rows], rotate=rotate)
    ko, vo = (torch.empty(rows, kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sv.spec_kv4_read(step, 1, ko, vo)
    raw = c.bytes()
    assert sum(O.negative_zeros(page, 2, kv, d) for page in raw) == 0
    want = O.stored(x[0].double().cpu().numpy(), x[1].double().cpu().numpy(),
                    range(3, 3 + rows) if rotate else None, 1e4)
    for got, w, from_ in zip((ko, vo), want, x.double().cpu().numpy()):
        assert ((w == 0) & (from_ < 0)).sum() > rows * kv * d / 20           # there are many
        bits = got.view(torch.int16).cpu().numpy()
        assert (bits[w == 0] == 0).all() and (bits[w != 0] != 0).all()


# ---- the same rows in other company ------------------------------------------------

def test_rows_alone_and_among_others():
    """A sample's rows by themselves, by one-row steps' kernels, and in batches whose other samples bring
    two row tiles per wave, split ranges or both: the same cache, keys and queries, so the outputs lie
    within their bound of each other's exact value."""
    cfg = config(8, 2, 128)
    kv, d, hq = 2, 128, 1024
    rng = np.random.default_rng(17)
    lens, rows = [129, 12000, 1, 700], [3, 5, 1, 90]
    for first in (3, 1):                                  # 12 rows per KV head; 4
        rows[0] = first
        c = Cache(cfg, lens, rows, seed=first)
        prefix = c.prefix(0)
        x = torch.from_numpy(rng.normal(size=(sum(rows), hq + 2 * kv * d))).to(torch.bfloat16).cuda()
        parents = [random_tree(rng, r) for r in rows]
        at = np.concatenate([[0], np.cumsum(rows)])
        outs, held = [], []
        for ids in ([0], [0, 1], [0, 2], [3, 0], [0, 1, 2, 3]):
            part = torch.cat([x[at[b]:at[b + 1]] for b in ids])
            step = sv.KV4Step(c.pool, ids, np.concatenate([[0], np.cumsum([rows[b] for b in ids])]),
                              sum((parents[b] for b in ids), []), [lens[b] for b in ids])
            sv.spec_kv4_append(step, 0, part[:, hq:hq + kv * d], part[:, hq + kv * d:])
            out = torch.empty(len(part), hq, dtype=torch.bfloat16, device="cuda")
            sv.spec_kv4_attend(step, 0, part[:, :hq], out)
            mine = sum(rows[b] for b in ids[:ids.index(0)])
            outs.append(out[mine:mine + first].double().cpu().numpy().reshape(first, 8, d))
            K, V = read(step, 0, len(part), kv, d)
            held.append((K[mine:mine + first], V[mine:mine + first]))
        for K, V in held[1:]:
            assert np.array_equal(K, held[0][0]) and np.array_equal(V, held[0][1])
        K, V = (np.concatenate([prefix[0][i], held[0][i]]) for i in (0, 1))
        visible = np.concatenate([np.ones((first, lens[0]), bool), O.sees(parents[0], first)[0]], 1)
        q = x[:first, :hq].double().cpu().numpy().reshape(first, 8, d)
        o, spread = O.attend(q, K, V, visible)
        tol = O.attend_bound(q, K, V, visible, o, spread)
        for out in outs:
            assert (np.abs(out - o) <= tol).all()
            assert (np.abs(out - outs[0]) <= 2 * tol).all()


@pytest.mark.parametrize("shape", [(8, 2, 128), (12, 4, 64)], ids=str)
def test_tree_equals_one_token_steps(shape):
    """The rows of a tree's branches, attended at once, and one at a time by one-row steps over the same
    prefix, each of which sees what the ones before it appended: the same numbers in the cache, outputs
    within their bound of one exact value."""
    cfg = config(*shape, theta=5e5)
    kv, d, hq = cfg.n_kv_heads, cfg.head_dim, cfg.n_heads * cfg.head_dim
    rng = np.random.default_rng(23)
    S, n = 203, 40
    parents = random_tree(rng, n)
    sees, depth = O.sees(parents, n)
    leaves = [i for i in range(n) if i not in parents][-3:] + [int(depth.argmax())]
    paths = [np.nonzero(sees[i])[0] for i in leaves]
    c = Cache(cfg, [S] * (1 + len(paths)), [n] * (1 + len(paths)), seed=2)
    p = torch.from_numpy(rng.normal(size=(2, S, kv, d)) * 1.3).to(torch.bfloat16).cuda()
    for b in range(1 + len(paths)):                       # one prefix for all
        step = c.append(0, [b], [0], p[0], p[1], [S])
    prefix = read(step, 0, S, kv, d)
    x = torch.from_numpy(rng.normal(size=(n, hq + 2 * kv * d)) * 1.3).to(torch.bfloat16).cuda()
    k, v = x[:, hq:hq + kv * d], x[:, hq + kv * d:]
    step = c.append(0, [0], [S], k, v, [n], parents)
    own = read(step, 0, n, kv, d)
    out = torch.empty(n, hq, dtype=torch.bfloat16, device="cuda")
    sv.spec_kv4_attend(step, 0, x[:, :hq], out)
    out = out.double().cpu().numpy().reshape(n, -1, d)
    for b, path in enumerate(paths, 1):
        for t, node in enumerate(path):
            row = x[node:node + 1]
            step = c.append(0, [b], [S + t], row[:, hq:hq + kv * d], row[:, hq + kv * d:], [1])
            K, V = read(step, 0, 1, kv, d)
            assert np.array_equal(K[0], own[0][node]) and np.array_equal(V[0], own[1][node])
            one = torch.empty(1, hq, dtype=torch.bfloat16, device="cuda")
            sv.spec_kv4_attend(step, 0, row[:, :hq], one)
            q = row[:, :hq].double().cpu().numpy().reshape(1, -1, d)
            K, V = (np.concatenate([prefix[i], own[i][path[:t + 1]]]) for i in (0, 1))
            seen = np.ones((1, S + t + 1), bool)
            o, spread = O.attend(q, K, V, seen)
            tol = O.attend_bound(q, K, V, seen, o, spread)[0]
            assert (np.abs(one.double().cpu().numpy().reshape(-1, d) - o[0]) <= tol).all()
            assert (np.abs(out[node] - o[0]) <= tol).all()


# ---- the element-wise bound over the kernel's shapes -----------------------------------

@pytest.mark.parametrize("shape,lens,rows,chain,std", [
    ((8, 2, 128), [500, 64], [8, 20], False, 8.0),        # scores of several hundred
    ((8, 2, 64), [500, 64], [8, 20], False, 8.0),
    ((8, 2, 128), [700], [40], False, 30.0),              # of several thousand
    ((32, 8, 128), [65, 0], [17, 9], False, 1.3),
    ((4, 2, 64), [0, 1, 63, 200], [1, 9, 33, 40], True, 1.3),
    ((3, 3, 128), [64, 130], [2, 70], True, 3.0),
    ((14, 2, 128), [257], [33], False, 3.0),
    ((8, 4, 64), [9001, 40], [3, 5], False, 3.0),         # split ranges
    ((8, 2, 128), [300], [400], True, 3.0),
], ids=str)
def test_attend_element_by_element(shape, lens, rows, chain, std):
    cfg = config(*shape)
    rng = np.random.default_rng(sum(rows))
    n, kv, d = sum(rows), cfg.n_kv_heads, cfg.head_dim
    hq = cfg.n_heads * d
    c = Cache(cfg, lens, rows, seed=n)
    prefix = c.prefix(0, std=std)
    parents = None if chain else [p for r in rows for p in random_tree(rng, r)]
    x = torch.from_numpy(rng.normal(size=(n, hq + 2 * kv * d)) * std).to(torch.bfloat16).cuda()
    step = c.append(0, range(len(lens)), lens, x[:, hq:hq + kv * d], x[:, hq + kv * d:], rows, parents)
    own = read(step, 0, n, kv, d)
    out = torch.full((n, hq), float("nan"), dtype=torch.bfloat16, device="cuda")
    sv.spec_kv4_attend(step, 0, x[:, :hq], out)
    q, out = (t.double().cpu().numpy().reshape(n, -1, d) for t in (x[:, :hq], out))
    at = 0
    for b, (s, r) in enumerate(zip(lens, rows)):
        sl = slice(at, at + r)
        at += r
        m, _ = O.sees(None if chain else parents[sl], r)
        check(q[sl], out[sl], *(np.concatenate([prefix[b][i], own[i][sl]]) for i in (0, 1)),
              np.concatenate([np.ones((r, s), bool), m], 1), f"sample {b}")


# ---- workspaces of just the bytes that a step needs -----------------------------------

@pytest.mark.parametrize("shape,lens,rows,chain", [
    ((8, 2, 128), [0], [1], True), ((8, 2, 128), [3000], [1], False), ((8, 2, 128), [3000, 5, 2900], [40, 1, 9], False),
    ((4, 2, 64), [20000], [33], True), ((32, 8, 128), [700, 3], [300, 2], True), ((8, 4, 64), [511, 512, 6000], [1, 1, 1], True),
], ids=str)
def test_workspace_of_exactly_the_step(shape, lens, rows, chain):
    """The bytes behind it stay as they are, and the attention is right."""
    cfg = config(*shape)
    rng = np.random.default_rng(len(lens))
    n, kv, d = sum(rows), cfg.n_kv_heads, cfg.head_dim
    hq = cfg.n_heads * d
    c = Cache(cfg, lens, rows)
    prefix = c.prefix(0)
    parents = None if chain else [p for r in rows for p in random_tree(rng, r)]
    need = sv.spec_kv4_step_bytes(cfg, len(lens), n, sum((s + r + 63) // 64 for s, r in zip(lens, rows)))
    whole = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    offsets = np.concatenate([[0], np.cumsum(rows)])
    with pytest.raises(sv.SpecError, match="workspace"):
        sv.KV4Step(c.pool, range(len(lens)), offsets, parents, lens, workspace=whole[:need - 1])
    step = sv.KV4Step(c.pool, range(len(lens)), offsets, parents, lens, workspace=whole[:need])
    x = torch.from_numpy(rng.normal(size=(n, hq + 2 * kv * d))).to(torch.bfloat16).cuda()
    sv.spec_kv4_append(step, 0, x[:, hq:hq + kv * d], x[:, hq + kv * d:])
    own = read(step, 0, n, kv, d)
    out = torch.empty(n, hq, dtype=torch.bfloat16, device="cuda")
    sv.spec_kv4_attend(step, 0, x[:, :hq], out)
    assert (whole[need:] == 0xA5).all()
    q, out = (t.double().cpu().numpy().reshape(n, -1, d) for t in (x[:, :hq], out))
    at = 0
    for b, (s, r) in enumerate(zip(lens, rows)):
        sl = slice(at, at + r)
        at += r
        m, _ = O.sees(None if chain else parents[sl], r)
        check(q[sl], out[sl], *(np.concatenate([prefix[b][i], own[i][sl]]) for i in (0, 1)),
              np.concatenate([np.ones((r, s), bool), m], 1), f"sample {b}")


def test_a_query_that_is_not_finite_is_its_rows_alone():
    """A NaN or infinity in one row and head: that row and head come out as NaN, the others as they do
    without it, in one tile and in two, with ranges that are split."""
    cfg = config(8, 2, 128)
    rng = np.random.default_rng(5)
    for lens, rows in (([40], [6]), ([9000, 3], [50, 2])):
        n = sum(rows)
        c = Cache(cfg, lens, rows)
        c.prefix(0)
        x = torch.from_numpy(rng.normal(size=(n, 1024 + 512))).to(torch.bfloat16).cuda()
        step = c.append(0, range(len(lens)), lens, x[:, 1024:1280], x[:, 1280:], rows,
                        [p for r in rows for p in random_tree(rng, r)])
        q = x[:, :1024].clone().view(n, 8, 128)
        plain, out = (torch.empty(n, 1024, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        sv.spec_kv4_attend(step, 0, q, plain)
        bad = torch.zeros(n, 8, dtype=torch.bool)
        for r, h, d, v in ((0, 3, 7, float("nan")), (4, 0, 127, float("inf")), (n - 1, 7, 64, float("-inf"))):
            q[r, h, d] = v
            bad[r, h] = True
        sv.spec_kv4_attend(step, 0, q, out)
        out, plain = out.view(n, 8, 128).cpu(), plain.view(n, 8, 128).cpu()
        assert torch.isfinite(plain).all() and torch.equal(out[~bad], plain[~bad])
        assert torch.isnan(out[bad]).all()
