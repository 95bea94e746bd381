"""GPU parity of the verify step over the 4-bit pool (spec_verify_kv4) against
the float64 oracle.

A key's code can differ from the oracle's where bf16 noise moves a number over
a midpoint, which no tolerance on logits covers.  So the comparison is in two
parts.  The K/V that the step stored, read back, lie within half a step of the
grid (plus the bf16 tolerance) of the oracle's.  And the logits equal, under the
element-wise rule of the bf16 cache's tests, those of the oracle when its
attention takes the stored K/V.
"""

import dataclasses
import sys

import numpy as np
import pytest
import torch

import oracle
import paper_2512_04752_amd as sv
import workload as wl
from oracle import sampling as SA
from tests.gpu_util import (ATOL, RTOL, check_argmax, check_logits, check_meta,
                            check_sample_acceptance, run_gpu, split_rows)

pytestmark = pytest.mark.gpu

OV = sys.modules["oracle.verify"]           # the module; oracle.verify is its function

CONFIGS = {
    "tiny": wl.TINY,
    "d128": wl.ModelConfig(2, 1024, 8, 2, 128, 2048, 1024, rope_theta=5e5),
    "g1": wl.ModelConfig(2, 256, 4, 4, 64, 1024, 1024),
}


def setup(cfg, caps, seed, max_tokens, sampling=False):
    W = wl.make_weights(cfg, seed)
    W_dev = {k: v.cuda() for k, v in W.items() if k != "layers"}
    W_dev["layers"] = [{k: v.cuda() for k, v in lw.items()} for lw in W["layers"]]
    return W, sv.Verifier(cfg, W_dev, caps, len(caps), max_tokens, sampling=sampling, cache="kv4")


def stored(ver, ids, lens, rows):
    """What the cache holds in slots [S, S + rows) of the samples: K, V [layers, kv heads, rows, d]."""
    cfg = ver.cfg
    out = []
    for i, s, r in zip(ids, lens, rows):
        if r == 0:
            out.append((torch.empty(cfg.n_layers, cfg.n_kv_heads, 0, cfg.head_dim, dtype=torch.float64),) * 2)
            continue
        step = sv.KV4Step(ver.kv, [i], [0, r], None, [s])
        kv = torch.empty(cfg.n_layers, 2, r, cfg.n_kv_heads, cfg.head_dim, dtype=torch.bfloat16, device="cuda")
        for l in range(cfg.n_layers):
            sv.spec_kv4_read(step, l, kv[l, 0], kv[l, 1])
        kv = kv.double().cpu().transpose(2, 3)
        out.append((kv[:, 0], kv[:, 1]))
    return out


def fill(ver, lens, seed):
    cfg = ver.cfg
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for b, s in enumerate(lens):
        if s == 0:
            continue
        step = sv.KV4Step(ver.kv, [b], [0, s], None, [0])
        for l in range(cfg.n_layers):
            kv = torch.empty(2, s, cfg.n_kv_heads, cfg.head_dim, dtype=torch.bfloat16, device="cuda")
            kv.normal_(0, wl.prefix_kv_std(cfg), generator=gen)
            sv.spec_kv4_append(step, l, kv[0], kv[1], rotate=False)


def check_verify(monkeypatch, cfg, W, ver, ids, trees, lens):
    out = run_gpu(ver, ids, trees, lens)
    rows = [len(t[0]) for t in trees]
    prefix = stored(ver, ids, [0] * len(ids), lens)
    own = stored(ver, ids, lens, rows)
    calls = []
    plain = OV.attention

    def on_stored(q, k_all, v_all, visible, n_kv_heads, rnd=OV._identity):
        l, b = divmod(len(calls), len(ids))
        calls.append((l, b))
        k = torch.cat([prefix[b][0][l], own[b][0][l]], 1)
        v = torch.cat([prefix[b][1][l], own[b][1][l]], 1)
        assert k.shape == k_all.shape
        return plain(q, k, v, visible, n_kv_heads, rnd)

    with monkeypatch.context() as m:
        m.setattr(OV, "attention", on_stored)
        r = oracle.verify(cfg, W, [p[0] for p in prefix], [p[1] for p in prefix], lens, trees)
    assert len(calls) == cfg.n_layers * len(ids)
    check_meta(trees, lens, out)
    # stored numbers: within half the widest step (2, below 6) of their group's grid
    for b in range(len(ids)):
        for got, want, group in ((own[b][0], r["tree_k"][b], 32), (own[b][1], r["tree_v"][b], cfg.head_dim)):
            top = want.reshape(*want.shape[:-1], -1, group).abs().amax(-1, keepdim=True)
            half = (top * (1 + RTOL) + ATOL) * 2 / 6       # a step is at most 2 * 2^e, 2^e < top / 3
            err = (got - want).abs().reshape(*top.shape[:-1], group)
            tol = half + ATOL + RTOL * want.abs().reshape(*top.shape[:-1], group)
            assert (err <= tol).all(), f"sample {b}: stored numbers off by up to {(err - tol).max()}"
    st = check_logits(out["logits"], r["logits"], "kv4")
    excused = check_argmax(out["argmax"], r["logits"], st["tie_tol"])
    offs, g = split_rows(trees), out["argmax"].tolist()
    g_or = r["argmax"].tolist()
    for b, (tokens, parents) in enumerate(trees):
        sl = slice(offs[b], offs[b + 1])
        check_sample_acceptance(tokens, parents, g[sl], out["accepted_len"][b], out["next_token"][b],
                                out["nodes"][b], r, b, g_or[sl],
                                [i - offs[b] for i in excused if offs[b] <= i < offs[b + 1]])
    return out, own


@pytest.mark.parametrize("name", sorted(CONFIGS))
def test_verify_and_commit(monkeypatch, name):
    """Three steps in a row, trees that follow the target's greedy choice so that branches are
    accepted; each step sees what the commits left."""
    cfg = CONFIGS[name]
    rng = np.random.default_rng(5)
    lens = [0, 130, 63, 700]
    W, ver = setup(cfg, [s + 200 for s in lens], 3, 160)
    fill(ver, lens, 1)
    ids = [2, 0, 3, 1]
    lens = [lens[i] for i in ids]
    for rows in ([9, 33, 1, 40], [5, 17, 8, 64], [1, 1, 2, 1]):
        trees = [(wl.random_tokens(rng, n, cfg.vocab), wl.recursive_tree(rng, n, min(n, 8), 4)) for n in rows]
        # greedy tokens of the first pass become drafts of the second, two levels deep
        for _ in range(2):
            g = run_gpu(ver, ids, trees, lens)["argmax"].tolist()
            offs = split_rows(trees)
            for b, (tok, par) in enumerate(trees):
                for i in range(1, len(tok)):
                    if par[i] not in par[1:i]:
                        tok[i] = int(g[offs[b] + par[i]])
        out, own = check_verify(monkeypatch, cfg, W, ver, ids, trees, lens)
        new = ver.commit(ids, lens).tolist()
        acc = out["accepted_len"]
        assert new == [s + a + 1 for s, a in zip(lens, acc)]
        moved = stored(ver, ids, lens, [a + 1 for a in acc])
        for b in range(len(ids)):
            path = out["nodes"][b][:acc[b] + 1].tolist()
            assert torch.equal(moved[b][0], own[b][0][:, :, path])
            assert torch.equal(moved[b][1], own[b][1][:, :, path])
        lens = new


def test_sampled_and_eos_over_kv4():
    """Acceptance at a temperature and with an EOS token runs on this pool's logits."""
    cfg = wl.TINY
    rng = np.random.default_rng(9)
    lens = [40, 129]
    W, ver = setup(cfg, [400, 400], 4, 64, sampling=True)
    fill(ver, lens, 2)
    trees = [(wl.random_tokens(rng, n, cfg.vocab), wl.recursive_tree(rng, n, 6, 4)) for n in (12, 20)]
    q = torch.softmax(torch.randn(32, cfg.vocab, generator=torch.Generator("cuda").manual_seed(1),
                                  device="cuda"), -1)
    u = torch.rand(32, 2, generator=torch.Generator("cuda").manual_seed(2), device="cuda")
    dbg = ver.debug_buffers(32)
    acc, nxt, nodes = ver.verify_sampled([0, 1], trees, lens, 1.0, draft_probs=q, uniforms=u, debug=dbg)
    torch.cuda.synchronize()
    offs = split_rows(trees)
    for b, (tok, par) in enumerate(trees):
        sl = slice(offs[b], offs[b + 1])
        a, n, path, margin = SA.sample_accept(tok, par, dbg["logits"][sl].double().cpu().numpy(), 1.0,
                                              q[sl].double().cpu().numpy(), u[sl].double().cpu().numpy())
        assert margin < 1e-11 or (int(acc[b]), int(nxt[b]), nodes[b, :a + 1].tolist()) == (a, n, path)
    eos = int(trees[0][0][0])
    acc, nxt, _ = ver.verify_sampled([0, 1], trees, lens, 0.0, eos_token=eos)
    assert (int(acc[0]), int(nxt[0])) == (0, -1)


def test_step_beyond_the_mapped_pages_is_refused():
    cfg = wl.TINY
    W, ver = setup(cfg, [64, 64], 4, 64)
    tree = ([1, 2, 3], [-1, 0, 0])
    with pytest.raises(sv.SpecError, match="CAPACITY"):
        ver.verify([0, 1], [tree, tree], [10, 62])
    ver.kv.map(1, [1, 0])                     # sample 0's page, shared: still read only
    with pytest.raises(sv.SpecError, match="mapped"):
        ver.verify([0], [tree], [10])
    with pytest.raises(ValueError):
        ver.verify_noalloc([0], [tree], [10])


def test_repeated_step_is_bitwise_the_same():
    cfg = dataclasses.replace(wl.TINY, n_heads=8, hidden=512)
    rng = np.random.default_rng(1)
    W, ver = setup(cfg, [600, 300], 6, 64)
    fill(ver, [500, 7], 3)
    trees = [(wl.random_tokens(rng, n, cfg.vocab), wl.recursive_tree(rng, n, min(n, 8), 4)) for n in (30, 10)]
    a = run_gpu(ver, [0, 1], trees, [500, 7])
    b = run_gpu(ver, [0, 1], trees, [500, 7])
    assert torch.equal(a["logits"], b["logits"])
