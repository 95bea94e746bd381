"""GPU parity of the cache rows that follow the beams, over both pools: every byte of the
pool as the oracle (oracle.drafting.reorder) has it."""

import numpy as np
import pytest
import torch

import paper_2512_04752_amd as sv
import workload as wl
from oracle import drafting as O
from oracle import kv4 as O4

pytestmark = pytest.mark.gpu
PAGE = sv.SPEC_KV4_PAGE


def config(kv_heads, d, layers):
    return wl.ModelConfig(layers, 256, kv_heads * 2, kv_heads, d, 256, 256)


def parents_of(rng, groups, width, kind):
    if kind == "cycle":                  # each takes the next one's
        p = (np.arange(width) + 1) % width
        return np.tile(p, (groups, 1))
    if kind == "one":                    # all take one beam's
        return np.tile(rng.integers(width, size=(groups, 1)), (1, width))
    if kind == "stay":
        return np.tile(np.arange(width), (groups, 1))
    p = rng.integers(width, size=(groups, width))
    if kind == "none":                   # and some have no candidate, or a number that is no beam
        p[rng.random((groups, width)) < 0.4] = -1
        p[0, 0] = width
        p[-1, -1] = 2 ** 31 - 1
    return p


KINDS = ["any", "cycle", "one", "stay", "none"]
# (the last shapes have more descriptors than go along as kernel arguments)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("kv_heads,d,layers,groups,width", [
    (2, 64, 1, 1, 1), (2, 64, 2, 3, 2), (1, 128, 2, 2, 8), (2, 64, 1, 2, 9), (3, 128, 1, 2, 17), (1, 128, 1, 2, 33),
    (2, 64, 1, 1, 64), (2, 64, 1, 60, 5), (2, 64, 1, 70, 2)], ids=str)
def test_bf16_pool(kv_heads, d, layers, groups, width, kind):
    rng = np.random.default_rng(width)
    cfg = config(kv_heads, d, layers)
    n = groups * width
    spare = 2
    caps = [int(c) for c in rng.integers(70, 90, size=n + spare)]
    pool = sv.KVPool(cfg, caps)
    pool.buf.copy_(torch.from_numpy(rng.integers(0, 256, size=pool.buf.numel(), dtype=np.uint8)))
    ids = rng.permutation(n + spare)[:n].reshape(groups, width)
    begin = rng.integers(0, 40, size=groups)
    end = begin + rng.integers(0, 30, size=groups)
    end[0], begin[-1] = 70, 0
    parents = parents_of(rng, groups, width, kind)
    used = max(sv.binding.spec_kv_sample_layout(pool.handle, s)[0] + layers * 2 * kv_heads * caps[s] * d * 2
               for s in range(n + spare))
    want = pool.buf[:used].clone()

    def views(buf, s):
        off, cap = sv.binding.spec_kv_sample_layout(pool.handle, s)
        return buf[off:off + layers * 2 * kv_heads * cap * d * 2].view(layers * 2 * kv_heads, cap, 2 * d)

    held = [[views(pool.buf, s)[:, begin[g]:end[g]].clone() for s in ids[g]] for g in range(groups)]
    for g, beams in enumerate(O.reorder(held, parents)):
        for j, x in enumerate(beams):
            views(want, ids[g][j])[:, begin[g]:end[g]] = x
    sv.spec_kv_reorder(pool, ids, begin, end, torch.from_numpy(parents.astype(np.int32)).cuda())
    torch.cuda.synchronize()
    assert torch.equal(pool.buf[:used], want)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("kv_heads,d,layers,groups,width,begin,end", [
    (2, 64, 1, 2, 2, 0, 1), (2, 64, 2, 3, 3, 5, 64), (1, 128, 2, 2, 8, 63, 65), (2, 64, 1, 1, 9, 64, 128),
    (2, 128, 1, 1, 17, 1, 200), (1, 128, 1, 1, 33, 130, 139), (2, 64, 1, 1, 64, 37, 100), (1, 128, 1, 2, 4, 70, 70),
    (2, 64, 1, 66, 2, 60, 70), (2, 64, 1, 23, 20, 3, 190)], ids=str)
def test_kv4_pool(kv_heads, d, layers, groups, width, begin, end, kind):
    """Each head's bytes, position by position, from the layout."""
    rng = np.random.default_rng(width + end)
    cfg = config(kv_heads, d, layers)
    n, per = groups * width, 4
    pool = sv.KV4Pool(cfg, n + 1, (n + 1) * per)
    pages = rng.permutation((n + 1) * per).reshape(n + 1, per)
    for s in range(n + 1):
        pool.map(s, pages[s])
    nbytes = sv.spec_kv4_page_bytes(cfg) * pool.n_pages
    pool.buf.copy_(torch.from_numpy(rng.integers(0, 256, size=pool.buf.numel(), dtype=np.uint8)))
    before = pool.buf[:nbytes].cpu().numpy().reshape(pool.n_pages, layers * kv_heads, -1)
    ids = rng.permutation(n + 1)[:n].reshape(groups, width)
    parents = parents_of(rng, groups, width, kind)
    begins, ends = np.full(groups, begin), np.full(groups, end)
    ends[-1] = min(ends[-1] + 3, per * PAGE)

    def nibbles(t):                      # of a head's bytes: (byte, low half) of position t's numbers
        at = [(t // 32 * 16 * d + c * 512 + t % 32 * 16 + i, h) for c in range(d // 32) for i in range(16) for h in (0, 1)]
        at += [(32 * d + t // 8 * 4 * d + w * 4 + t % 8 // 2, t % 2) for w in range(d)]
        for base, per_pos in ((64 * d, d // 32), (64 * (d + d // 32), 2)):
            at += [(base + t * per_pos + i, h) for i in range(per_pos) for h in (0, 1)]
        return at

    masks = []                           # [64 positions, head bytes]
    for t in range(PAGE):
        m = np.zeros(before.shape[2], np.uint8)
        for byte, high in nibbles(t):
            m[byte] |= 0xF0 if high else 0x0F
        masks.append(m)
    assert (np.bitwise_or.reduce(masks) == 255).all()
    want = before.copy()
    for g in range(groups):
        for p in range(begins[g] // PAGE, -(-ends[g] // PAGE) if begins[g] < ends[g] else 0):
            mask = np.zeros(before.shape[2], np.uint8)
            for t in range(max(0, begins[g] - p * PAGE), min(PAGE, ends[g] - p * PAGE)):
                mask |= masks[t]
            held = [[before[pages[s][p]] for s in ids[g]]]
            for j, x in enumerate(O.reorder(held, parents[g:g + 1])[0]):
                page = pages[ids[g][j]][p]
                want[page] = (before[page] & ~mask) | (x & mask)
    sv.spec_kv4_reorder(pool, ids, begins, ends, torch.from_numpy(parents.astype(np.int32)).cuda())
    torch.cuda.synchronize()
    got = pool.buf[:nbytes].cpu().numpy().reshape(before.shape)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("n_pages,pages", [(65536, [65535, 0]), (65600, [65599, 65536])], ids=str)
def test_high_page_ids(n_pages, pages):
    """Page ids take 16 bits where they go along as kernel arguments: not in a pool of more."""
    cfg = config(2, 64, 1)
    pool = sv.KV4Pool(cfg, 2, n_pages)
    held = pool.buf[:sv.spec_kv4_page_bytes(cfg) * n_pages].view(n_pages, -1)
    held.zero_()
    for s, p in enumerate(pages):
        pool.map(s, [p])
        held[p] = s + 1
    sv.spec_kv4_reorder(pool, [[0, 1]], [0], [PAGE], torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"))
    assert (held[pages[0]] == 2).all() and (held[pages[1]] == 1).all()
    assert int(held.long().sum()) == 3 * held.shape[1]


def test_far_block_of_the_bf16_pool():
    """A sample whose block begins past 4 GB."""
    cfg = config(8, 128, 16)
    cap = 1 + (1 << 32) // (cfg.n_layers * 2 * cfg.n_kv_heads * cfg.head_dim * 2)
    pool = sv.KVPool(cfg, [cap, 8, 8])
    want = []
    for s in (1, 2):
        k, v = pool.sample_view(s)
        k.normal_()
        v.normal_()
        want.append((k.clone(), v.clone()))
    sv.spec_kv_reorder(pool, [[1, 2]], [2], [7], torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"))
    for s in (1, 2):
        for got, own, other in zip(pool.sample_view(s), want[s - 1], want[2 - s]):
            assert torch.equal(got[:, :, 2:7], other[:, :, 2:7])
            assert torch.equal(got[:, :, :2], own[:, :, :2]) and torch.equal(got[:, :, 7:], own[:, :, 7:])


def test_refusals():
    cfg = config(2, 64, 1)
    kv, kv4 = sv.KVPool(cfg, [100] * 4), sv.KV4Pool(cfg, 4, 8)
    for s in range(4):
        kv4.map(s, [2 * s, 2 * s + 1])
    p = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    ids = [[0, 1], [2, 3]]
    for pool, call in ((kv, sv.spec_kv_reorder), (kv4, sv.spec_kv4_reorder)):
        for bad in ((ids, [0], [1, 1], p), (ids, [0, 0], [1, 1], p.cpu()), (ids, [0, 0], [1, 1], p[:1]),
                    (ids, [0, 0], [1, 1], p.long()), ([0, 1, 2, 3], [0, 0], [1, 1], p)):
            with pytest.raises(ValueError):
                call(pool, *bad)
        for bad in ((ids, [0, -1], [1, 1]), (ids, [0, 2], [1, 1]), (ids, [0, 0], [1, 129]), ([[0, 1], [2, 4]], [0, 0], [1, 1]),
                    ([[0, 1], [1, 3]], [0, 0], [1, 1])):
            with pytest.raises(sv.SpecError):
                call(pool, *bad, p)
        with pytest.raises(sv.SpecError, match="captured"):
            side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                torch.zeros(1, device="cuda")
                call(pool, ids, [0, 0], [1, 1], p)
    kv4.map(1, [0, 3])                   # page 0 is sample 0's too
    with pytest.raises(sv.SpecError, match="mapped to 2"):
        sv.spec_kv4_reorder(kv4, ids, [0, 0], [1, 1], p)
    sv.spec_kv4_reorder(kv4, ids, [64, 0], [65, 1], p)
    with pytest.raises(ValueError, match="workspace"):
        sv.spec_kv4_reorder(kv4, ids, [64, 0], [65, 1], p, workspace=torch.empty(256, device="cuda"))
    torch.cuda.synchronize()
