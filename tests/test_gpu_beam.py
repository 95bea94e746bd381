"""GPU parity of the choice of beams against the float64 oracle (oracle.drafting):
the same parents and tokens in the same order, and scores.  An exponential is off by at
most 3e-10 of itself (its series' next term is (ln 2 / 2)^9 / 9! = 2e-10), so a sum of
them by 3e-10 of itself and its logarithm by 3e-10; the doubles' own roundings are below
1e-13 (2^-53 of numbers below 500, a few times).  A score is rounded to fp32 once: half a
step, 2^-24 of it."""

import numpy as np
import pytest
import torch

import paper_2512_04752_amd as sv
from oracle import drafting as O

pytestmark = pytest.mark.gpu
INF = float("inf")


def run(z, s, k, last=None, eos=-1, **kw):
    groups, width = z.shape[:2]
    parents, tokens = (torch.full((groups, k), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    new = torch.full((groups, k), 7.0, device="cuda")
    sv.spec_beam_select(z, s, parents, tokens, new, last_tokens=last, eos_token=eos, **kw)
    return parents, tokens, new


def check(z, s, k, last=None, eos=-1, got=None, **kw):
    got = got or run(z, s, k, last, eos, **kw)
    want = O.select(z.double().cpu().numpy(), s.double().cpu().numpy(), k, None if last is None else last.tolist(), eos)
    assert got[0].tolist() == want[0].tolist()
    assert got[1].tolist() == want[1].tolist()
    new = got[2].double().cpu().numpy()
    none = want[2] == -np.inf
    assert np.array_equal(new == -np.inf, none)
    new, exact = new[~none], want[2][~none]
    assert (np.abs(new - exact) <= 2.0 ** -24 * np.abs(exact) + 3.1e-10).all()


def logits(seed, groups, width, vocab, dtype=torch.float32, std=2.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(groups, width, vocab, device="cuda").normal_(0, std, generator=gen).to(dtype)


def scores(seed, groups, width):
    gen = torch.Generator(device="cuda").manual_seed(seed + 1000)
    return -torch.empty(groups, width, device="cuda").uniform_(0, 8, generator=gen)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("groups,width,vocab,k", [
    (1, 1, 1, 1), (1, 1, 5, 3), (3, 2, 63, 7), (2, 5, 64, 64), (1, 4, 257, 4), (4, 8, 1000, 8), (1, 64, 300, 64),
    (2, 64, 1025, 1), (1, 1, 32001, 17), (5, 3, 4099, 33), (2, 12, 50001, 24), (1, 1, 128256, 64), (9, 7, 8192, 10),
    (70, 9, 515, 9), (40, 30, 8001, 20)])
def test_select(groups, width, vocab, k, dtype):
    """bf16 logits bring many equal ones within a beam: the lower token first."""
    z = logits(vocab + k, groups, width, vocab, dtype)
    check(z, scores(k, groups, width), k)


@pytest.mark.parametrize("std", [0.01, 0.3, 30.0, 3000.0])
def test_flat_and_sharp(std):
    check(logits(1, 3, 6, 9001, std=std), scores(1, 3, 6), 12)


@pytest.mark.parametrize("order", ["up", "down", "equal", "saw"])
@pytest.mark.parametrize("k", [1, 5, 64])
def test_orders(order, k):
    """Every logit enters the list (rising), none but the first (falling), or all are equal."""
    n = 6000
    ramp = torch.arange(n, dtype=torch.float32, device="cuda") / 1024
    z = {"up": ramp, "down": -ramp, "equal": torch.full((n,), 1.5, device="cuda"),
         "saw": (torch.arange(n, device="cuda") % 7).float()}[order]
    check(z.expand(2, 3, n).contiguous(), torch.tensor([[0.0, -1.0, 0.5]] * 2, device="cuda"), k)


def test_equal_beams():
    """Beams with the same logits and scores, in rows that start at different alignments."""
    z = logits(5, 1, 1, 4999).expand(3, 6, 4999).contiguous()
    check(z, torch.zeros(3, 6, device="cuda"), 20)
    check(z.to(torch.bfloat16), torch.zeros(3, 6, device="cuda"), 20)


def test_masked_tokens_and_beams():
    z = logits(2, 4, 4, 700)
    z[0, :, 100:] = -INF                 # most tokens masked
    z[1, 2] = -INF                       # a beam with no token
    z[2] = -INF                          # a group without a candidate
    z[3, :, 3:] = -INF                   # fewer candidates than k
    s = scores(2, 4, 4)
    s[0, 1] = -INF
    s[1, 0] = -INF
    check(z, s, 16)
    lowest = torch.finfo(torch.float32).min
    z = logits(3, 2, 3, 900)
    z[0, :, 50:] = lowest                # masked by the type's lowest value
    z[1, 1] = lowest                     # and everywhere: as good as uniform
    z[0, 2, :3], z[0, 2, 3:] = lowest, -INF
    check(z, scores(3, 2, 3), 8)


def test_infinities_and_nan_take_their_beam_out():
    z, s = logits(4, 3, 4, 1500), scores(4, 3, 4)
    z[0, 1, 1499] = float("nan")
    z[0, 2, 7] = INF
    z[1, 3, 0], z[1, 3, 900] = -INF, INF
    s[1, 1], s[2, 0], s[2, 3] = float("nan"), INF, -INF
    check(z, s, 9)


def test_large_logits():
    """Far beyond the range of an exponential, rising by thousands along a row."""
    z = logits(6, 2, 3, 3001, std=1.0)
    z[0] += 1e5
    z[1] += torch.arange(3001, device="cuda") * 50.0 - 2e4
    z[1, 2, 5] = 3e38
    check(z, scores(6, 2, 3), 6)


def test_beams_that_have_ended():
    z, s = logits(7, 5, 6, 320), scores(7, 5, 6)
    eos = 319
    last = torch.randint(0, 300, (5, 6), dtype=torch.int32, device="cuda")
    last[0, 2] = last[1, 0] = last[1, 5] = eos
    last[2] = eos                        # all: fewer candidates than k
    last[3, 1] = eos
    s[3, 1] = -INF
    z[0, 2] = float("nan")               # not read
    check(z, s, 8, last, eos)
    check(z, s, 8, last, -1)             # no end of sequence


def test_strided_logits():
    big = logits(8, 4, 3, 2050)
    check(big[:, :, 1:2000], scores(8, 4, 3), 5)
    half = big.to(torch.bfloat16)
    check(half[:, :, 3:2001], scores(8, 4, 3), 5)
    check(half[:, 1:2], scores(8, 4, 1), 5)
    check(big[1:2, :, :77], scores(8, 1, 3), 5)


def test_in_place_outputs_graph_and_streams():
    """A loop's own use: scores and last tokens replaced in place, replayed."""
    groups, width, vocab = 6, 5, 3000
    z = logits(9, groups, width, vocab)
    s, last = scores(9, groups, width), torch.zeros(groups, width, dtype=torch.int32, device="cuda")
    parents = torch.empty_like(last)
    ws = torch.empty(sv.spec_beam_workspace_bytes(groups, width, vocab, width), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sv.spec_beam_select(z, s, parents, last, s, last_tokens=last, eos_token=11, workspace=ws)
    for step in range(4):
        z.copy_(logits(20 + step, groups, width, vocab))
        z[:, :, 11] += 6.0
        before = s.clone(), last.clone()
        ws.fill_(step)
        graph.replay()
        torch.cuda.synchronize()
        check(z, before[0], width, before[1], 11, got=(parents, last, s))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(z, s, 7, stream=side)
    torch.cuda.synchronize()
    check(z, s, 7, got=got)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("k", [9, 24, 64])
def test_segments_that_share_their_bounds(k, dtype):
    """More than 8 of a long row: its waves leave out what the others' bounds rule out, so rows
    whose candidates lie in one segment, or nowhere, or all at one value."""
    groups, width, vocab, eos = 8, 3, 9001, 17
    z, s = logits(k, groups, width, vocab, dtype), scores(k, groups, width)
    lowest = torch.finfo(dtype).min
    z[0, :, 500:] = -INF                 # all in the first segment
    z[1, :, :8900] = -INF                # all in the last
    z[2, :, 5:] = -INF                   # fewer than k
    z[3, :, 3000:] = lowest
    z[3, 1] = lowest
    z[4, 0] = 2.5                        # ties over all segments
    z[4, 1, ::2] = 7.0
    z[5, 0, 4000], z[5, 1, 8999] = float("nan"), INF
    z[6] = -INF
    z[6, 1, ::1000] = 1.0
    z[7, 0] += torch.arange(vocab, device="cuda").to(dtype) * 0.25
    last = torch.zeros(groups, width, dtype=torch.int32, device="cuda")
    last[0, 1] = last[5, 2] = eos
    check(z, s, k, last, eos)
    check(z, s, k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_graph_with_shared_bounds(dtype):
    groups, width, vocab = 3, 12, 7000
    z, s = logits(9, groups, width, vocab, dtype), scores(9, groups, width)
    last = torch.zeros(groups, width, dtype=torch.int32, device="cuda")
    parents = torch.empty_like(last)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sv.spec_beam_select(z, s, parents, last, s)
    for step in range(4):
        z.copy_(logits(30 + step, groups, width, vocab, dtype))
        before = s.clone()
        graph.replay()
        torch.cuda.synchronize()
        check(z, before, width, got=(parents, last, s))


def test_refusals_of_tensors():
    z, s = logits(1, 2, 3, 100), scores(1, 2, 3)
    i32 = dict(dtype=torch.int32, device="cuda")
    ok = dict(logits=z, scores=s, parents=torch.empty(2, 4, **i32), tokens=torch.empty(2, 4, **i32),
              new_scores=torch.empty(2, 4, device="cuda"))
    for bad in (dict(logits=z.half()), dict(logits=z.cpu()), dict(logits=z[0]), dict(logits=z[:, :, ::2]),
                dict(logits=z.transpose(0, 1)[:, :2]), dict(scores=s[:1]), dict(scores=s.double()), dict(scores=s.cpu()),
                dict(parents=torch.empty(2, 5, **i32)), dict(tokens=torch.empty(2, 4, device="cuda")),
                dict(new_scores=torch.empty(2, 4, dtype=torch.float64, device="cuda")),
                dict(last_tokens=torch.empty(2, 4, **i32), eos_token=1)):
        with pytest.raises(ValueError):
            sv.spec_beam_select(**{**ok, **bad})
    for bad in (dict(eos_token=1), dict(eos_token=100, last_tokens=torch.empty(2, 3, **i32)), dict(eos_token=-2),
                dict(workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(sv.SpecError):
            sv.spec_beam_select(**{**ok, **bad})
