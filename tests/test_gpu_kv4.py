"""GPU parity of the 4-bit paged KV cache against the float64 oracle
(oracle.kv4): appended rows, their bytes, attention, and commits.

What the cache holds is compared exactly: the rotation is computed in doubles
on both sides, and a code differs only where a rotated number lies within about
1e-15 of a midpoint between codes.

Attention is compared element-wise with a bound made of its roundings.  With
A = sum softmax |V|, o the exact output and u = 2^-8 (half a step of bf16,
relative): the probabilities' rounding gives at most u A, the output's u |o|.
In fp32 (v = 2^-24): a score is a sum of d products whose rounding errors are at
most (d + 2) v sum |q k| / sqrt(d) =: (d + 2) v B, plus 4 v |score| <= 4 v B for
the scale and the subtraction of the maximum; exp2 adds 4 v (its argument's
last bit counted in B); each enters the numerator and the denominator, so
2 ((d + 6) v B + 4 v) A.  Sums over the n visible keys and the merges of their
parts: 2 (n + 70) v A.  Numbers below 2^-126 may be flushed to zero: a probability
(at most 2^-126 |V| lost, the row's sum being at least 1), its product with the
value's power of two (whose code is at most 6) and the output, together
(n + 1) 2^-126 (max |V| + 6).  A query number enters as a sum of e4m3 parts: off by at
most 2^-17 of its row's largest where it is more than 2^10 below that one, by 2^-34 of it
in a row whose largest is above 32 times its mean; a score so by that times
sum |k| / sqrt(d) at most, the output by 2 A of it (added where rows have outliers).
"""

import numpy as np
import pytest
import torch

import paper_2512_04752_amd as sv
import workload as wl
from oracle import kv4 as O

pytestmark = pytest.mark.gpu

PAGE = sv.SPEC_KV4_PAGE


def config(heads, kv_heads, d, layers=1, theta=1e4):
    return wl.ModelConfig(layers, 256, heads, kv_heads, d, 256, 256, rope_theta=theta)


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16)


class Cache:
    """A pool with scattered pages per sample, first filled with one byte value."""

    def __init__(self, cfg, lens, rows, fill=0xFF, spare=1, seed=0):
        self.cfg, self.lens = cfg, list(lens)
        need = [(s + r + PAGE - 1) // PAGE + spare for s, r in zip(lens, rows)]
        order = np.random.default_rng(seed).permutation(sum(need) + 1)[1:]
        self.pool = sv.KV4Pool(cfg, len(need), sum(need) + 1)
        self.pool.buf.fill_(fill)
        self.pages = np.split(order, np.cumsum(need)[:-1])
        for b, p in enumerate(self.pages):
            self.pool.map(b, p)

    def append(self, layer, ids, lens, k, v, rows, parents=None, rotate=True):
        step = sv.KV4Step(self.pool, ids, np.concatenate([[0], np.cumsum(rows)]), parents, lens)
        sv.spec_kv4_append(step, layer, k, v, rotate=rotate)
        return step

    def prefix(self, layer, std=1.3, seed=1):
        """Random committed K/V of every sample (as already rotated); returns what is stored."""
        ids = [b for b, s in enumerate(self.lens) if s]
        got = [(np.empty((0, self.cfg.n_kv_heads, self.cfg.head_dim)),) * 2] * len(self.lens)
        if not ids:
            return got
        n = sum(self.lens)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        k, v = (torch.empty(n, self.cfg.n_kv_heads, self.cfg.head_dim, dtype=torch.bfloat16,
                            device="cuda").normal_(0, std, generator=gen) for _ in range(2))
        step = self.append(layer, ids, [0] * len(ids), k, v, [self.lens[b] for b in ids], rotate=False)
        ko, vo = torch.empty_like(k), torch.empty_like(v)
        sv.spec_kv4_read(step, layer, ko, vo)
        at = 0
        for b in ids:
            got[b] = tuple(x[at:at + self.lens[b]].double().cpu().numpy() for x in (ko, vo))
            at += self.lens[b]
        return got

    def bytes(self):
        torch.cuda.synchronize()
        n = sv.spec_kv4_page_bytes(self.cfg) * self.pool.n_pages
        return self.pool.buf[:n].cpu().numpy().reshape(self.pool.n_pages, -1)


def random_tree(rng, n, kids=4):
    p = [-1]
    for i in range(1, n):
        p.append(int(rng.integers(max(0, i - kids), i)))
    return p


def positions(lens, rows, parents):
    pos, at = [], 0
    for s, r in zip(lens, rows):
        par = None if parents is None else parents[at:at + r]
        pos += [s + int(x) for x in O.sees(par, r)[1]]
        at += r
    return pos


def same_numbers(got, want):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    bad = np.nonzero(~np.isnan(want) & (got != want))
    assert len(bad[0]) == 0, f"{len(bad[0])} numbers differ, first at {[x[0] for x in bad]}: " \
                             f"{got[tuple(x[0] for x in bad)]} not {want[tuple(x[0] for x in bad)]}"


# ---- append and read ---------------------------------------------------------

SHAPES = [(4, 2, 64), (2, 1, 128), (32, 8, 128), (12, 4, 64), (3, 3, 128)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("kind", ["one", "octet_ends", "tree", "run", "strided", "rotated_already"])
def test_append_and_read(shape, kind):
    """Values, exactly; the page bytes, decoded by the layout's definition, hold the same; all
    other bytes of the pool stay as they were."""
    cfg = config(*shape, layers=2, theta=5e5)
    rng = np.random.default_rng(7)
    lens, rows = {"one": ([63], [1]), "octet_ends": ([0, 1, 7, 8, 60, 64], [8, 6, 1, 1, 9, 3]),
                  "tree": ([100, 3], [31, 12]), "run": ([0, 70], [70, 200])}.get(kind, ([5, 62], [11, 4]))
    n, kv, d = sum(rows), cfg.n_kv_heads, cfg.head_dim
    parents = None if kind == "run" else [p for r in rows for p in random_tree(rng, r)]
    c = Cache(cfg, lens, rows, fill=0x5A)
    before = c.bytes().copy()
    wide = torch.from_numpy(rng.normal(size=(n, 2 * kv * d + 24))).to(torch.bfloat16).cuda()
    if kind == "strided":
        k, v = wide[:, 8:8 + kv * d].view(n, kv, d), wide[:, 16 + kv * d:16 + 2 * kv * d]
    else:
        k, v = wide[:, :kv * d].reshape(n, kv, d), wide[:, kv * d:2 * kv * d].reshape(n, kv, d)
    rotate = kind != "rotated_already"
    step = c.append(1, range(len(lens)), lens, k, v, rows, parents, rotate)
    out = torch.full((n, 2 * kv * d + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    ko, vo = out[:, :kv * d].view(n, kv, d), out[:, 8 + kv * d:]
    sv.spec_kv4_read(step, 1, ko, vo)
    torch.cuda.synchronize()
    want = O.stored(k.double().cpu().numpy(), v.reshape(n, kv, d).double().cpu().numpy(),
                    positions(lens, rows, parents) if rotate else None, 5e5)
    same_numbers(ko, want[0])
    same_numbers(vo.reshape(n, kv, d), want[1])
    assert (out[:, kv * d:kv * d + 8] == 7).all()

    after = c.bytes()
    assert np.array_equal(after[:, :before.shape[1] // 2], before[:, :before.shape[1] // 2])   # layer 0
    at = 0
    for b, (s, r) in enumerate(zip(lens, rows)):
        for i, p in enumerate(c.pages[b]):
            K, V = O.decode_page(after[p], 2, kv, d)
            K0, V0 = O.decode_page(before[p], 2, kv, d)
            for t in range(PAGE):
                row = i * PAGE + t - s
                if 0 <= row < r:
                    assert np.array_equal(K[1, :, t], want[0][at + row])
                    assert np.array_equal(V[1, :, t], want[1][at + row])
                else:
                    assert np.array_equal(K[:, :, t], K0[:, :, t], equal_nan=True)
                    assert np.array_equal(V[:, :, t], V0[:, :, t], equal_nan=True)
        at += r
    unused = sorted(set(range(c.pool.n_pages)) - set(np.concatenate(c.pages).tolist()))
    assert np.array_equal(after[unused], before[unused])


@pytest.mark.parametrize("d", [64, 128])
def test_midpoints_and_ends_of_the_range(d):
    """Every midpoint between codes, its neighbours, both signs, at exponents over the whole range
    of bf16; zeros; groups with an infinity or NaN."""
    cfg = config(256 // d, 256 // d, d)
    kv = cfg.n_kv_heads
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    near = np.concatenate([mids, mids * (1 + 2 ** -7), mids * (1 - 2 ** -7), [0.0, 6.0, 4.5, 5.5]])
    near = np.concatenate([near, -near])                       # 50 numbers
    rows = []
    for e in (-133, -127, -126, -125, -60, -1, 0, 1, 77, 124, 125):
        for top in (6.0, 6.0 * (1 + 2 ** -7), 4.0, 3.0 * (1 + 2 ** -7)):
            x = np.resize(near, kv * d)
            x[::16] = top
            rows.append(x * 2.0 ** e)
    rows += [np.zeros(kv * d), -np.zeros(kv * d)]
    for bad in (np.inf, -np.inf, np.nan):
        x = np.resize(near, kv * d)
        x[33] = bad
        rows.append(x)
    x = bf16(np.stack(rows)).view(-1, kv, d)
    c = Cache(cfg, [3], [len(x)])
    step = c.append(0, [0], [3], x.cuda(), x.cuda(), [len(x)], rotate=False)
    ko, vo = torch.empty_like(x, device="cuda"), torch.empty_like(x, device="cuda")
    sv.spec_kv4_read(step, 0, ko, vo)
    want = O.stored(x.double().numpy(), x.double().numpy())
    same_numbers(ko, want[0])
    same_numbers(vo, want[1])
    raw = c.bytes()[c.pages[0][0]]
    assert not np.isin(8, np.concatenate([raw[:64 * d // 2] & 15, raw[:64 * d // 2] >> 4])[:1]).any()
    assert (ko[-5:-3].view(torch.int16) == 0).all()            # zeros read as +0


@pytest.mark.parametrize("top", [1e38, 2.0 ** -140])
def test_rotated_extremes(top):
    """Rotation of the largest and smallest numbers: what is past 6 * 2^125 takes it, sqrt(2) times the
    largest bf16 (past fp32) too."""
    cfg = config(2, 1, 128)
    rng = np.random.default_rng(3)
    x = bf16(np.where(rng.random((40, 1, 128)) < 0.5, 1, -1) * top * 3.3).cuda()
    c = Cache(cfg, [1000], [40])
    step = c.append(0, [0], [1000], x, x, [40])
    ko, vo = torch.empty_like(x), torch.empty_like(x)
    sv.spec_kv4_read(step, 0, ko, vo)
    want = O.stored(x.double().cpu().numpy(), x.double().cpu().numpy(), range(1000, 1040), 1e4)
    same_numbers(ko, want[0])
    same_numbers(vo, want[1])


# ---- attention ---------------------------------------------------------------

def check_attend(cfg, q, out, prefix, own, lens, rows, parents, samples=None, q_off=0.0):
    at = 0
    d = cfg.head_dim
    q = q.double().cpu().numpy().reshape(-1, cfg.n_heads, d)
    out = out.double().cpu().numpy().reshape(q.shape)
    for b, (s, r) in enumerate(zip(lens, rows)):
        sl = slice(at, at + r)
        at += r
        if samples is not None and b not in samples:
            continue
        m, _ = O.sees(None if parents is None else parents[sl], r)
        K, V = (np.concatenate([prefix[b][i], own[i][sl]]) for i in (0, 1))
        o, A = O.attend(q[sl], K, V, np.concatenate([np.ones((r, s), bool), m], 1))
        B = max(np.abs(q[sl]).max(axis=(0, 1)) @ np.abs(K).max(axis=(0, 1)), 1.0) / np.sqrt(d)
        v = 2.0 ** -24
        tol = 2.0 ** -8 * (A + np.abs(o)) + (2 * ((d + 6) * v * B + 4 * v) + 2 * (s + r + 70) * v) * A
        tol = tol + (s + r + 1) * 2.0 ** -126 * (np.abs(V).max() + 6)
        tol = tol + 2 * q_off * np.abs(q[sl]).max() * np.abs(K).sum(-1).max() / np.sqrt(d) * A
        err = np.abs(out[sl] - o)
        assert (err <= tol).all(), f"sample {b}: error {err.max()} over {(err - tol).max()} past its bound"


def attend_case(shape, lens, rows, chain, seed=0, layers=2, samples=None, std=1.3):
    cfg = config(*shape, layers=layers)
    rng = np.random.default_rng(seed)
    layer = layers - 1
    c = Cache(cfg, lens, rows, seed=seed)
    prefix = c.prefix(layer, std=std, seed=seed + 1)
    n, kv, d = sum(rows), cfg.n_kv_heads, cfg.head_dim
    parents = None if chain else [p for r in rows for p in random_tree(rng, r)]
    x = torch.from_numpy(rng.normal(size=(n, (cfg.n_heads + 2 * kv) * d)) * std).to(torch.bfloat16).cuda()
    hq = cfg.n_heads * d
    k, v = x[:, hq:hq + kv * d], x[:, hq + kv * d:]
    step = c.append(layer, range(len(lens)), lens, k, v, rows, parents)
    ko, vo = (torch.empty(n, kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sv.spec_kv4_read(step, layer, ko, vo)
    out = torch.full((n, hq), float("nan"), dtype=torch.bfloat16, device="cuda")
    sv.spec_kv4_attend(step, layer, x[:, :hq], out)
    again = torch.empty_like(out)
    sv.spec_kv4_attend(step, layer, x[:, :hq], again)
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    own = tuple(t.double().cpu().numpy() for t in (ko, vo))
    check_attend(cfg, x[:, :hq], out, prefix, own, lens, rows, parents, samples)


@pytest.mark.parametrize("shape", [(4, 2, 64), (32, 8, 128), (2, 1, 128), (16, 2, 64), (3, 3, 128), (6, 2, 64),
                                   (14, 2, 128)], ids=str)
@pytest.mark.parametrize("kind", ["tree", "run"])
def test_attend_head_layouts(shape, kind):
    """Query heads per KV head 1, 2, 3, 4, 7, 8; row tiles cut inside a node; no committed keys, pages that
    end inside a block, row counts around the tile groups."""
    attend_case(shape, [0, 1, 63, 64, 65, 200], [1, 9, 33, 2, 17, 40], kind == "run", seed=3)


@pytest.mark.parametrize("rows", [1, 8, 9, 16, 17, 32, 33, 63, 64, 65, 129, 256])
def test_attend_tree_sizes(rows):
    """One to 256 nodes, 4 query heads to a KV head: 1, 2 and up to 4 row tiles per work-group, with
    ranges that are split."""
    attend_case((8, 2, 128), [700, 5], [rows, max(1, rows // 2)], False, seed=rows)


@pytest.mark.parametrize("shape", [(8, 2, 128), (8, 4, 64)], ids=str)
@pytest.mark.parametrize("length", [255, 256, 257, 4095, 9001])
def test_attend_split_ranges(shape, length):
    attend_case(shape, [length, 40], [3, 5], False, seed=length)


def test_attend_long_run():
    """A prompt's piece of 700 rows behind 300 cached ones: causal masks across row groups."""
    attend_case((8, 2, 128), [300, 0], [700, 260], True, seed=5)


def test_attend_many_samples():
    rng = np.random.default_rng(9)
    lens = rng.integers(0, 900, size=70).tolist()
    rows = rng.integers(1, 12, size=70).tolist()
    attend_case((8, 2, 64), lens, rows, False, seed=9, samples=set(range(0, 70, 7)))


def test_attend_large_scores():
    """Scores of several hundred: one key takes all."""
    attend_case((8, 2, 128), [500, 64], [8, 20], False, seed=11, std=8.0)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [5, 40, 90])
def test_attend_queries_with_outliers(d, rows):
    """Rows of which one number dwarfs the others, in a dimension where the keys are zero; rows of tiny
    numbers, of zeros, and ordinary ones between them, which come out as they do without those."""
    cfg = config(8, 2, d)
    rng = np.random.default_rng(rows)
    c = Cache(cfg, [0], [rows])
    k = bf16(rng.normal(size=(rows, 2, d)))
    k[:, :, 5] = 0
    v = bf16(rng.normal(size=(rows, 2, d))).cuda()
    step = c.append(0, [0], [0], k.cuda(), v, [rows], rotate=False)
    ko, vo = (torch.empty(rows, 2, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sv.spec_kv4_read(step, 0, ko, vo)
    assert (ko[:, :, 5] == 0).all()
    plain = rng.normal(size=(rows, 8, d))
    q = plain.copy()
    q[::3, :, 5] = 5000.0
    q[1::6] *= 2.0 ** -100
    q[1::6, :, 5] = 2.0 ** -80
    q[4::6] = 0
    out, alone = (torch.empty(rows, 8, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sv.spec_kv4_attend(step, 0, bf16(q).cuda(), out)
    sv.spec_kv4_attend(step, 0, bf16(plain).cuda(), alone)
    assert torch.equal(out[2::3], alone[2::3])
    own = tuple(t.double().cpu().numpy() for t in (ko, vo))
    none = [(np.empty((0, 2, d)),) * 2]
    check_attend(cfg, bf16(q), out, none, own, [0], [rows], None, q_off=2.0 ** -34)


def test_attend_at_32k_keys():
    attend_case((4, 1, 128), [32701], [20], False, seed=2, layers=1)


def test_unseen_keys_do_not_matter():
    """Slots past the rows and other branches' keys may hold anything, infinities and NaN among them."""
    cfg = config(8, 2, 128)
    rng = np.random.default_rng(4)
    kv, d, hq = 2, 128, 1024
    parents = [-1, 0, 0, 1, 2]
    x = torch.from_numpy(rng.normal(size=(5, hq + 2 * kv * d))).to(torch.bfloat16).cuda()
    outs = []
    for fill, poison in ((0xFF, False), (0x00, False), (0x33, True)):
        c = Cache(cfg, [37], [5], fill=fill)
        c.prefix(0)
        k, v = x[:, hq:hq + kv * d].clone(), x[:, hq + kv * d:].clone()
        if poison:                                  # node 2's keys: nodes 2 and 4 see them
            k[2, 5] = float("inf")
            v[2, 140] = float("nan")
        step = c.append(0, [0], [37], k, v, [5], parents)
        out = torch.empty(5, hq, dtype=torch.bfloat16, device="cuda")
        sv.spec_kv4_attend(step, 0, x[:, :hq], out)
        outs.append(out.float().cpu().view(5, 2, 4, d))
    assert torch.equal(outs[0], outs[1])
    clean = [0, 1, 3]
    assert torch.equal(outs[0][clean], outs[2][clean])
    assert torch.isfinite(outs[0]).all()
    for i in (2, 4):
        assert not torch.isfinite(outs[2][i, 0]).all(-1).any()      # head 0: its K
        assert not torch.isfinite(outs[2][i, 1]).any()              # head 1: its V row


def test_rows_in_any_batch_give_the_same():
    """A sample's rows alone and among others: the same keys, within two roundings of each other."""
    attend_case((8, 2, 128), [129], [6], False, seed=21)
    attend_case((8, 2, 128), [129, 2000, 1], [6, 30, 1], False, seed=21)


# ---- pages -------------------------------------------------------------------

def test_shared_prefix_pages():
    """Three samples share two pages of a prompt; their own rows go to their own pages."""
    cfg = config(8, 2, 128)
    rng = np.random.default_rng(6)
    S, rows = 128, [5, 9, 1]
    kv, d, hq = 2, 128, 1024
    pool = sv.KV4Pool(cfg, 4, 8)
    pool.buf.fill_(0xFF)
    pool.map(3, [6, 2])
    p = torch.from_numpy(rng.normal(size=(2, S, kv, d))).to(torch.bfloat16).cuda()
    prompt = sv.KV4Step(pool, [3], [0, S], None, [0])
    sv.spec_kv4_append(prompt, 0, p[0], p[1])
    po = torch.empty_like(p)
    sv.spec_kv4_read(prompt, 0, po[0], po[1])
    for b, own in enumerate((0, 7, 3)):
        pool.map(b, [6, 2, own])
    with pytest.raises(sv.SpecError):
        sv.KV4Step(pool, [3], [0, 1], None, [S - 1])
    parents = [x for r in rows for x in random_tree(rng, r)]
    x = torch.from_numpy(rng.normal(size=(15, hq + 2 * kv * d))).to(torch.bfloat16).cuda()
    step = sv.KV4Step(pool, [0, 1, 2], [0, 5, 14, 15], parents, [S] * 3)
    sv.spec_kv4_append(step, 0, x[:, hq:hq + kv * d], x[:, hq + kv * d:])
    ko, vo = (torch.empty(15, kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sv.spec_kv4_read(step, 0, ko, vo)
    out = torch.empty(15, hq, dtype=torch.bfloat16, device="cuda")
    sv.spec_kv4_attend(step, 0, x[:, :hq], out)
    prefix = [tuple(po.double().cpu().numpy())] * 3
    check_attend(cfg, x[:, :hq], out, prefix, tuple(t.double().cpu().numpy() for t in (ko, vo)),
                 [S] * 3, rows, parents)


def test_offsets_past_32_bits():
    """The last pages of a pool of 5 GB, the last of 32 layers."""
    cfg = config(32, 8, 128, layers=32)
    n_pages = 5 * 2 ** 30 // sv.spec_kv4_page_bytes(cfg)
    pool = sv.KV4Pool(cfg, 2, n_pages)
    pool.map(0, [n_pages - 1, 0, n_pages - 2])
    pool.map(1, [1])
    rng = np.random.default_rng(8)
    kv, d, hq = 8, 128, 4096
    prefix = []
    for b, s in enumerate((130, 20)):
        p = torch.from_numpy(rng.normal(size=(2, s, kv, d))).to(torch.bfloat16).cuda()
        step = sv.KV4Step(pool, [b], [0, s], None, [0])
        sv.spec_kv4_append(step, 31, p[0], p[1], rotate=False)
        sv.spec_kv4_read(step, 31, p[0], p[1])
        prefix.append(tuple(p.double().cpu().numpy()))
    x = torch.from_numpy(rng.normal(size=(3, hq + 2 * kv * d))).to(torch.bfloat16).cuda()
    step = sv.KV4Step(pool, [0, 1], [0, 2, 3], [-1, 0, -1], [130, 20])
    sv.spec_kv4_append(step, 31, x[:, hq:hq + kv * d], x[:, hq + kv * d:])
    ko, vo = (torch.empty(3, kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sv.spec_kv4_read(step, 31, ko, vo)
    out = torch.empty(3, hq, dtype=torch.bfloat16, device="cuda")
    sv.spec_kv4_attend(step, 31, x[:, :hq], out)
    check_attend(cfg, x[:, :hq], out, prefix, tuple(t.double().cpu().numpy() for t in (ko, vo)),
                 [130, 20], [2, 1], [-1, 0, -1])


# ---- commit ------------------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
def test_commit_moves_rows(d):
    """Random bit patterns in every page; branches of every kind: whole chains (nothing moves), jumps,
    the deepest ids, branches past the pages' end; bytes of other positions stay."""
    kv, layers = 256 // d, 3
    cfg = config(kv, kv, d, layers=layers)
    lens = [0, 5, 61, 64, 200, 33, 100]
    c = Cache(cfg, lens, [256] * 7, spare=0, seed=d)
    rng = np.random.default_rng(d)
    raw = rng.integers(0, 256, size=c.pool.buf.numel(), dtype=np.uint8)
    c.pool.buf.copy_(torch.from_numpy(raw))
    before = c.bytes().copy()
    paths = [list(range(256)), [0, 255], [0, 3, 5, 6, 9, 20, 21, 70, 255], [0],
             sorted(rng.choice(np.arange(1, 256), 100, replace=False).tolist()), [0, 1, 2, 200],
             [0, 254, 255]]
    paths[4] = [0] + paths[4]
    nodes = np.full((7, 256), -1, np.int32)
    for b, p in enumerate(paths):
        nodes[b, :len(p)] = p
    acc = torch.tensor([len(p) - 1 for p in paths], dtype=torch.int32, device="cuda")
    new = torch.zeros(7, dtype=torch.int32, device="cuda")
    ids = [3, 0, 6, 1, 2, 5, 4]
    sv.spec_kv4_commit(c.pool, ids, [lens[b] for b in ids], acc[ids].contiguous(),
                       torch.from_numpy(nodes[ids]).cuda(), new)
    after = c.bytes()
    assert new.tolist() == [lens[b] + len(paths[b]) for b in ids]
    for b, path in enumerate(paths):
        whole = [[np.concatenate([O.decode_page(x[p], layers, kv, d)[i] for p in c.pages[b]], axis=2)
                  for i in (0, 1)] for x in (before, after)]
        for i in (0, 1):
            want = whole[0][i].copy()
            for e, node in enumerate(path):
                want[:, :, lens[b] + e] = whole[0][i][:, :, lens[b] + node]
            assert np.array_equal(whole[1][i], want, equal_nan=True), (b, i)


def test_commit_clamps():
    """A depth past the pages' end, a negative one, node ids out of range: nothing is read or written
    outside the sample's pages."""
    cfg = config(4, 4, 64)
    c = Cache(cfg, [60, 100, 3], [4, 28, 1], spare=0)
    rng = np.random.default_rng(0)
    c.pool.buf.copy_(torch.from_numpy(rng.integers(0, 256, size=c.pool.buf.numel(), dtype=np.uint8)))
    before = c.bytes().copy()
    acc = torch.tensor([200, -7, 2], dtype=torch.int32, device="cuda")
    nodes = torch.full((3, 256), 999, dtype=torch.int32, device="cuda")
    nodes[2, :3] = torch.tensor([0, 1, -5], dtype=torch.int32)
    new = torch.zeros(3, dtype=torch.int32, device="cuda")
    sv.spec_kv4_commit(c.pool, [0, 1, 2], [60, 100, 3], acc, nodes, new)
    assert np.array_equal(c.bytes(), before)
    assert new.tolist() == [64, 101, 6]


# ---- streams, graphs, refusals -------------------------------------------------

def _small(seed=0):
    cfg = config(8, 2, 128)
    rng = np.random.default_rng(seed)
    c = Cache(cfg, [150, 10], [6, 3], seed=seed)
    prefix = c.prefix(0, seed=seed + 5)
    parents = [-1, 0, 0, 1, 2, 4, -1, 0, 1]
    x = torch.from_numpy(rng.normal(size=(9, 1024 + 512))).to(torch.bfloat16).cuda()
    step = sv.KV4Step(c.pool, [0, 1], [0, 6, 9], parents, [150, 10])
    return cfg, c, prefix, parents, x, step


def test_other_stream():
    cfg, c, prefix, parents, x, step = _small(1)
    ko, vo = (torch.empty(9, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    out = torch.empty(9, 1024, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    sv.spec_kv4_append(step, 0, x[:, 1024:1280], x[:, 1280:], stream=s)
    sv.spec_kv4_read(step, 0, ko, vo, stream=s)
    sv.spec_kv4_attend(step, 0, x[:, :1024], out, stream=s)
    s.synchronize()
    check_attend(cfg, x[:, :1024], out, prefix, tuple(t.double().cpu().numpy() for t in (ko, vo)),
                 [150, 10], [6, 3], parents)


def test_step_made_on_another_stream():
    """Steps that are planned, run and dropped on a side stream, while memory is freed and taken on the
    current one: their workspaces are the side stream's."""
    cfg, c, prefix, parents, x, _ = _small(4)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    want = None
    for i in range(6):
        busy = torch.full((1 << 26,), 0xFF, dtype=torch.uint8, device="cuda")
        del busy
        step = sv.KV4Step(c.pool, [0, 1], [0, 6, 9], parents, [150, 10], stream=s)
        assert step._made_on == s.cuda_stream
        out = torch.empty(9, 1024, dtype=torch.bfloat16, device="cuda")
        s.wait_stream(torch.cuda.current_stream())
        sv.spec_kv4_append(step, 0, x[:, 1024:1280], x[:, 1280:], stream=s)
        sv.spec_kv4_attend(step, 0, x[:, :1024], out, stream=s)
        del step
        s.synchronize()
        want = out if want is None else want
        assert torch.equal(out, want)


def test_captured_and_replayed():
    """append, read and attend in a graph, replayed on new inputs, with eager work between the replays."""
    cfg, c, prefix, parents, x, step = _small(2)
    ko, vo = (torch.empty(9, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    out = torch.empty(9, 1024, dtype=torch.bfloat16, device="cuda")

    def run():
        sv.spec_kv4_append(step, 0, x[:, 1024:1280], x[:, 1280:])
        sv.spec_kv4_read(step, 0, ko, vo)
        sv.spec_kv4_attend(step, 0, x[:, :1024], out)

    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
        with pytest.raises(sv.SpecError, match="captured"):
            sv.KV4Step(c.pool, [0], [0, 1], None, [150], workspace=step.workspace)
    for seed in range(4):
        x.copy_(torch.from_numpy(np.random.default_rng(seed).normal(size=x.shape)).to(torch.bfloat16))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (ko, vo, out)]
        run()
        torch.cuda.synchronize()
        for a, b in zip(got, (ko, vo, out)):
            assert torch.equal(a, b)
        check_attend(cfg, x[:, :1024], out, prefix, tuple(t.double().cpu().numpy() for t in (ko, vo)),
                     [150, 10], [6, 3], parents)


def test_two_steps_on_one_pool():
    """Two planned steps with workspaces of their own, their launches interleaved."""
    cfg = config(8, 2, 128)
    rng = np.random.default_rng(12)
    c = Cache(cfg, [90, 300], [4, 7], seed=12)
    prefix = c.prefix(0)
    x = torch.from_numpy(rng.normal(size=(11, 1024 + 512))).to(torch.bfloat16).cuda()
    a = sv.KV4Step(c.pool, [0], [0, 4], None, [90])
    b = sv.KV4Step(c.pool, [1], [0, 7], None, [300])
    ko, vo = (torch.empty(11, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    out = torch.empty(11, 1024, dtype=torch.bfloat16, device="cuda")
    for step, sl in ((a, slice(0, 4)), (b, slice(4, 11))):
        sv.spec_kv4_append(step, 0, x[sl, 1024:1280], x[sl, 1280:])
    for step, sl in ((b, slice(4, 11)), (a, slice(0, 4))):
        sv.spec_kv4_read(step, 0, ko[sl], vo[sl])
        sv.spec_kv4_attend(step, 0, x[sl, :1024], out[sl])
    check_attend(cfg, x[:, :1024], out, prefix, tuple(t.double().cpu().numpy() for t in (ko, vo)),
                 [90, 300], [4, 7], None)


def test_launch_refusals():
    cfg, c, prefix, parents, x, step = _small(3)
    before = c.bytes().copy()
    k, v, q = x[:, 1024:1280], x[:, 1280:], x[:, :1024]
    out = torch.empty(9, 1024, dtype=torch.bfloat16, device="cuda")
    for layer in (-1, 1):
        with pytest.raises(sv.SpecError, match="layer"):
            sv.spec_kv4_append(step, layer, k, v)
        with pytest.raises(sv.SpecError, match="layer"):
            sv.spec_kv4_attend(step, layer, q, out)
    odd = torch.empty(9, 261, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(sv.SpecError, match="stride"):
        sv.spec_kv4_append(step, 0, odd[:, :256], v)
    with pytest.raises(sv.SpecError, match="aligned"):
        sv.spec_kv4_append(step, 0, k, torch.empty(9, 272, dtype=torch.bfloat16, device="cuda")[:, 4:260])
    for bad in (k.float(), k[:8], k.cpu(), x[:, 1024:1270], k.T):
        with pytest.raises(ValueError):
            sv.spec_kv4_append(step, 0, bad, v)
    with pytest.raises(ValueError):
        sv.spec_kv4_attend(step, 0, q, torch.empty(9, 2048, dtype=torch.bfloat16, device="cuda")[:, :1024])
    with pytest.raises(ValueError):
        sv.KV4Step(c.pool, [0, 1], [0, 6, 9], parents[:5], [150, 10])
    with pytest.raises(sv.SpecError, match="workspace"):
        sv.KV4Step(c.pool, [0, 1], [0, 6, 9], parents, [150, 10], workspace=step.workspace[:4096])
    for bad in (torch.empty(1 << 26, dtype=torch.int32, device="cuda"), torch.empty(1 << 26, dtype=torch.uint8),
                torch.empty(2, 1 << 26, dtype=torch.uint8, device="cuda")[:, ::2]):
        with pytest.raises(ValueError, match="workspace"):
            sv.KV4Step(c.pool, [0, 1], [0, 6, 9], parents, [150, 10], workspace=bad)
    lens, new = (torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(2))
    nodes = torch.zeros(2, sv.SPEC_MAX_TREE, dtype=torch.int32, device="cuda")
    for a, b, d in ((lens.cpu(), nodes, new), (lens.long(), nodes, new), (lens, nodes[:, ::2], new),
                    (lens, nodes[:1], new), (lens, nodes, new[:1])):
        with pytest.raises(ValueError):
            sv.spec_kv4_commit(c.pool, [0, 1], [150, 10], a, b, d)
    assert np.array_equal(c.bytes(), before)
    c.pool.close()
    with pytest.raises(ValueError, match="closed"):
        sv.spec_kv4_append(step, 0, k, v)


# ---- together ------------------------------------------------------------------

def test_prompt_trees_and_commits():
    """A prompt in two pieces, then trees, each committed along a branch: after every commit the next
    step sees exactly the accepted rows."""
    cfg = config(12, 4, 64, layers=2, theta=5e5)
    rng = np.random.default_rng(31)
    kv, d, hq = 4, 64, 12 * 64
    c = Cache(cfg, [0, 0], [200, 230], spare=1, seed=31)
    lens = [0, 0]
    held = [[[np.empty((0, kv, d))] * 2 for _ in range(2)] for _ in range(2)]     # [layer][sample][K, V]
    rounds = [("run", [100, 30]), ("run", [7, 90])] + [("tree", [9, 16])] * 3
    for kind, rows in rounds:
        n = sum(rows)
        parents = None if kind == "run" else [p for r in rows for p in random_tree(rng, r)]
        step = sv.KV4Step(c.pool, [0, 1], [0, rows[0], n], parents, lens)
        new = []
        for layer in range(2):
            x = torch.from_numpy(rng.normal(size=(n, hq + 2 * kv * d)) * 1.5).to(torch.bfloat16).cuda()
            sv.spec_kv4_append(step, layer, x[:, hq:hq + kv * d], x[:, hq + kv * d:])
            out = torch.empty(n, hq, dtype=torch.bfloat16, device="cuda")
            sv.spec_kv4_attend(step, layer, x[:, :hq], out)
            own = O.stored(x[:, hq:hq + kv * d].double().cpu().numpy().reshape(n, kv, d),
                           x[:, hq + kv * d:].double().cpu().numpy().reshape(n, kv, d),
                           positions(lens, rows, parents), 5e5)
            check_attend(cfg, x[:, :hq], out, held[layer], own, lens, rows, parents)
            new.append(own)
        paths = []
        for b, r in enumerate(rows):
            at = sum(rows[:b])
            path = list(range(r))
            if kind == "tree":
                path, node = [], int(rng.integers(r // 2, r))
                while node >= 0:
                    path.insert(0, node)
                    node = parents[at + node]
            paths.append(path)
            for layer in range(2):
                held[layer][b] = [np.concatenate([held[layer][b][i], new[layer][i][at:at + r][path]])
                                  for i in (0, 1)]
        if kind == "tree":
            nodes = torch.full((2, 256), -1, dtype=torch.int32)
            for b, p in enumerate(paths):
                nodes[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
            acc = torch.tensor([len(p) - 1 for p in paths], dtype=torch.int32, device="cuda")
            got = torch.zeros(2, dtype=torch.int32, device="cuda")
            sv.spec_kv4_commit(c.pool, [0, 1], lens, acc, nodes.cuda(), got)
            assert got.tolist() == [lens[b] + len(paths[b]) for b in range(2)]
        lens = [lens[b] + len(paths[b]) for b in range(2)]
