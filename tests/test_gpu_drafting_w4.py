"""Beam search over a model whose verify steps have weights in 4 bits: the step's logits, the
choice of beams and the cache that follows them, over both pools."""

import numpy as np
import pytest
import torch

import paper_2512_04752_amd as sv
import workload as wl
from oracle import drafting as O

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("groups,width", [(2, 3), (1, 16), (5, 8)])
@pytest.mark.parametrize("cache", ["bf16", "kv4"])
def test_beam_search(cache, groups, width):
    """Every choice is the oracle's on the logits at hand.  A beam's last logits are, bit for bit,
    those of its own tokens one after the other without beams."""
    cfg, steps, eos = wl.TINY, 6, 7
    n = groups * width
    weights = sv.W4Weights(wl.make_weights(cfg, 11, device="cuda"))
    rng = np.random.default_rng(4)
    prompt = rng.integers(0, cfg.vocab, size=(groups, 5))

    def session():
        ver = sv.Verifier(cfg, weights, [80] * n, max_batch=n, max_tokens=n, cache=cache, weights="w4")
        dbg = ver.debug_buffers(n)

        def feed(tokens, at):
            ver.verify(list(range(n)), [([int(t)], [-1]) for t in tokens], [at] * n, debug=dbg)
            ver.commit(list(range(n)), [at] * n)
            return dbg["logits"]

        for i in range(prompt.shape[1]):
            logits = feed(np.repeat(prompt[:, i], width), i)
        return ver, feed, logits

    reorder = sv.spec_kv_reorder if cache == "bf16" else sv.spec_kv4_reorder
    ver, feed, logits = session()
    scores = torch.full((groups, width), -float("inf"), device="cuda")
    scores[:, 0] = 0.0
    last = torch.full((groups, width), -1, dtype=torch.int32, device="cuda")
    parents = torch.empty_like(last)
    sequences = [[] for _ in range(n)]
    begin = prompt.shape[1]
    for t in range(steps):
        z = logits.view(groups, width, cfg.vocab)
        before, ends = scores.clone(), last.clone()
        sv.spec_beam_select(z, scores, parents, last, scores, last_tokens=last, eos_token=eos)
        want = O.select(z.double().cpu().numpy(), before.double().cpu().numpy(), width, ends.tolist(), eos)
        assert parents.tolist() == want[0].tolist() and last.tolist() == want[1].tolist()
        reorder(ver.kv, np.arange(n).reshape(groups, width), [begin] * groups, [begin + t] * groups, parents)
        sequences = [sequences[g * width + p] + [y] for g in range(groups) for p, y in zip(want[0][g], want[1][g])]
        logits = feed(last.view(-1).tolist(), begin + t)
    got = logits.clone()
    _, feed, _ = session()
    for t in range(steps):
        logits = feed([s[t] for s in sequences], begin + t)
    assert torch.equal(logits, got)
