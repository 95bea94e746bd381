"""The drafting operators as a loop uses them, one after the other: 4-bit products give
hidden states and logits, beams are chosen from them, and the cache follows the beams."""

import numpy as np
import pytest
import torch

import paper_2512_04752_amd as sv
import workload as wl
from oracle import drafting as O

pytestmark = pytest.mark.gpu


def test_draft_model_over_the_4bit_pool():
    """A decoder layer with 4-bit weights over the 4-bit pool, beams as its samples.  Every
    choice is the oracle's on the logits at hand, and after every step each beam's cache
    reads as the rows of its own history."""
    groups, width, prompt, steps, eos = 3, 4, 70, 9, 5
    cfg = wl.ModelConfig(1, 256, 4, 2, 64, 512, 640)
    n, d, kv = groups * width, cfg.head_dim, cfg.n_kv_heads
    hq, hk = cfg.n_heads * d, kv * d
    gen = torch.Generator(device="cuda").manual_seed(3)

    def normal(*shape, std=1.0):
        return torch.empty(shape, device="cuda").normal_(0, std, generator=gen)

    def matrix(rows, cols, std=0.05):
        return sv.W4Matrix(normal(rows, cols, std=std).bfloat16())

    qkv, o = matrix(hq + 2 * hk, cfg.hidden), matrix(cfg.hidden, hq)
    gate, up, down = matrix(cfg.ffn, cfg.hidden), matrix(cfg.ffn, cfg.hidden), matrix(cfg.hidden, cfg.ffn)
    head = matrix(cfg.vocab, cfg.hidden, std=0.15)
    embed = normal(cfg.vocab, cfg.hidden).bfloat16()
    pool = sv.KV4Pool(cfg, n, 3 * n)
    for b in range(n):
        pool.map(b, range(3 * b, 3 * b + 3))
    ids = np.arange(n).reshape(groups, width)

    def rows_of(step, k, v):
        sv.spec_kv4_read(step, 0, k, v)
        return torch.cat((k, v), 1).float().cpu().numpy()

    # a prompt that a group's beams share
    pk, pv = (normal(groups, 1, prompt, kv, d).expand(-1, width, -1, -1, -1).reshape(n * prompt, kv, d).bfloat16()
              for _ in range(2))
    step = sv.KV4Step(pool, range(n), np.arange(n + 1) * prompt, None, [0] * n)
    sv.spec_kv4_append(step, 0, pk, pv)

    scores = torch.full((groups, width), -float("inf"), device="cuda")
    scores[:, 0] = 0.0                       # one beam to begin with
    last = torch.full((groups, width), 7, dtype=torch.int32, device="cuda")
    parents = torch.empty_like(last)
    history = [[] for _ in range(n)]
    k_out, v_out = (torch.empty(n, kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in range(steps):
        x = embed[last.view(-1).long()]
        rows = torch.empty(n, hq + 2 * hk, dtype=torch.bfloat16, device="cuda")
        sv.spec_w4_linear(qkv, x, rows)
        step = sv.KV4Step(pool, range(n), range(n + 1), None, [prompt + t] * n)
        sv.spec_kv4_append(step, 0, rows[:, hq:hq + hk], rows[:, hq + hk:])
        attn = torch.empty(n, hq, dtype=torch.bfloat16, device="cuda")
        sv.spec_kv4_attend(step, 0, rows[:, :hq], attn)
        h = x.float()
        sv.spec_w4_linear(o, attn, h, add=True)
        act = torch.empty(n, cfg.ffn, dtype=torch.bfloat16, device="cuda")
        sv.spec_w4_gate_up(gate, up, h.bfloat16(), act)
        sv.spec_w4_linear(down, act, h, add=True)
        logits = torch.empty(n, cfg.vocab, device="cuda")
        sv.spec_w4_linear(head, h.bfloat16(), logits)
        for b, r in enumerate(rows_of(step, k_out, v_out)):
            history[b].append(r)
        z = logits.view(groups, width, cfg.vocab)
        before, ends = scores.clone(), last.clone()
        sv.spec_beam_select(z, scores, parents, last, scores, last_tokens=last, eos_token=eos)
        sv.spec_kv4_reorder(pool, ids, [prompt] * groups, [prompt + t + 1] * groups, parents)
        want = O.select(z.double().cpu().numpy(), before.double().cpu().numpy(), width, ends.tolist(), eos)
        assert parents.tolist() == want[0].tolist() and last.tolist() == want[1].tolist()
        assert np.isfinite(scores.cpu().numpy()).all()
        history = [history[g * width + p] for g, row in enumerate(want[0]) for p in row]
        history = [list(x) for x in history]
        # all the rows since the prompt, of every beam
        every = sv.KV4Step(pool, range(n), np.arange(n + 1) * (t + 1), None, [prompt] * n)
        k, v = (torch.empty(n * (t + 1), kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        got = rows_of(every, k, v).reshape(n, t + 1, -1)
        for b in range(n):
            assert np.array_equal(got[b], np.stack(history[b]).reshape(t + 1, -1))
    first = sv.KV4Step(pool, range(n), np.arange(n + 1) * prompt, None, [0] * n)
    a, b = (torch.empty_like(pk) for _ in range(4 // 2))
    sv.spec_kv4_read(first, 0, a, b)         # the prompt is as it was
    a = a.view(groups, width, prompt, kv, d)
    assert torch.equal(a, a[:, :1].expand_as(a))


@pytest.mark.parametrize("cache", ["bf16", "kv4"])
def test_beam_search_with_verify_steps(cache):
    """Beam search over the target model: one-node verify steps give the logits.  A beam's last
    logits are, bit for bit, those of its own tokens one after the other without beams."""
    cfg, groups, width, steps = wl.TINY, 2, 3, 6
    n = groups * width
    W = wl.make_weights(cfg, 11, device="cuda")
    rng = np.random.default_rng(4)
    prompt = rng.integers(0, cfg.vocab, size=(groups, 5))

    def session():
        return sv.Verifier(cfg, W, [64] * n, max_batch=n, max_tokens=n, cache=cache)

    def feed(ver, tokens, at, dbg):
        trees = [([int(t)], [-1]) for t in tokens]
        ver.verify(list(range(n)), trees, [at] * n, debug=dbg)
        ver.commit(list(range(n)), [at] * n)
        return dbg["logits"]

    reorder = sv.spec_kv_reorder if cache == "bf16" else sv.spec_kv4_reorder
    ver = session()
    dbg = ver.debug_buffers(n)
    for i in range(prompt.shape[1]):
        logits = feed(ver, np.repeat(prompt[:, i], width), i, dbg)
    scores = torch.full((groups, width), -float("inf"), device="cuda")
    scores[:, 0] = 0.0
    parents, tokens = (torch.empty(groups, width, dtype=torch.int32, device="cuda") for _ in range(2))
    sequences = [[] for _ in range(n)]
    begin = prompt.shape[1]
    for t in range(steps):
        z = logits.view(groups, width, cfg.vocab)
        before = scores.clone()
        sv.spec_beam_select(z, scores, parents, tokens, scores)
        want = O.select(z.double().cpu().numpy(), before.double().cpu().numpy(), width)
        assert parents.tolist() == want[0].tolist() and tokens.tolist() == want[1].tolist()
        reorder(ver.kv, np.arange(n).reshape(groups, width), [begin] * groups, [begin + t] * groups, parents)
        sequences = [sequences[g * width + p] + [y] for g in range(groups)
                     for p, y in zip(want[0][g], want[1][g])]
        logits = feed(ver, tokens.view(-1).tolist(), begin + t, dbg)
    got = logits.clone()
    alone = session()
    dbg = alone.debug_buffers(n)
    for i in range(prompt.shape[1]):
        feed(alone, np.repeat(prompt[:, i], width), i, dbg)
    for t in range(steps):
        logits = feed(alone, [s[t] for s in sequences], begin + t, dbg)
    assert torch.equal(logits, got)


def test_product_and_choice_in_one_graph():
    """The head's product and the choice, captured together and replayed over new states."""
    groups, width, hidden, vocab = 2, 5, 256, 3001
    gen = torch.Generator(device="cuda").manual_seed(9)
    head = sv.W4Matrix(torch.empty(vocab, hidden, device="cuda").normal_(0, 0.1, generator=gen).bfloat16())
    x = torch.empty(groups * width, hidden, dtype=torch.bfloat16, device="cuda")
    logits = torch.empty(groups * width, vocab, device="cuda")
    scores = torch.zeros(groups, width, device="cuda")
    parents, tokens = (torch.empty(groups, 7, dtype=torch.int32, device="cuda") for _ in range(2))
    new = torch.empty(groups, 7, device="cuda")

    def both():
        sv.spec_w4_linear(head, x, logits)
        sv.spec_beam_select(logits.view(groups, width, vocab), scores, parents, tokens, new)

    x.normal_(0, 1, generator=gen)
    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(4):
        x.normal_(0, 1, generator=gen)
        scores.uniform_(-3, 0, generator=gen)
        both()
        want = [t.clone() for t in (logits, parents, tokens, new)]
        for t in (logits, parents, tokens, new):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((logits, parents, tokens, new), want))
        chosen = O.select(logits.view(groups, width, vocab).double().cpu().numpy(), scores.double().cpu().numpy(), 7)
        assert parents.tolist() == chosen[0].tolist() and tokens.tolist() == chosen[1].tolist()
