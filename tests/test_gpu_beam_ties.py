"""Choices between continuations whose scores fp64 cannot tell apart, although their logits
differ: behind scores so large that logits are lost in them, or between logits so small that
they are lost in the normaliser.  The lower (beam, token) of equal scores comes first, as in
the float64 oracle."""

import pytest
import torch

import paper_2512_04752_amd as sv
from tests.test_gpu_beam import INF, check, logits, run

pytestmark = pytest.mark.gpu
LOWEST = torch.finfo(torch.float32).min
TYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
SIZES = pytest.mark.parametrize("groups,width,vocab,k", [
    (1, 1, 300, 1), (2, 3, 257, 5), (3, 4, 9001, 4), (2, 12, 20001, 24), (1, 64, 700, 64), (4, 2, 5000, 64), (40, 20, 1500, 7)])


def masked(z):
    """Tokens that are no candidates, the first ones among them."""
    z[:, :, :3] = -INF
    z[:, :, 10:200:2] = -INF
    return z


@TYPES
@SIZES
@pytest.mark.parametrize("score", [1e30, -1e30, LOWEST])
def test_scores_that_swallow_the_logits(groups, width, vocab, k, dtype, score):
    z = masked(logits(vocab, groups, width, vocab, dtype))
    check(z, torch.full((groups, width), score, device="cuda"), k)


@TYPES
@SIZES
def test_scores_that_swallow_parts_of_the_logits(groups, width, vocab, k, dtype):
    """Steps of 2^-13 between scores, some thousandths between logits."""
    z = masked(logits(vocab, groups, width, vocab, dtype, std=0.001))
    check(z, torch.full((groups, width), 1e12, device="cuda"), k)


@TYPES
@SIZES
def test_logits_that_vanish_beside_the_normaliser(groups, width, vocab, k, dtype):
    z = masked(logits(vocab, groups, width, vocab, dtype, std=1e-25))
    z[:, -1:, 5:9] = 2.0                     # and some that do not
    check(z, torch.zeros(groups, width, device="cuda"), k)


@TYPES
def test_dead_beams_at_the_lowest_score(dtype):
    """Few tokens are left to the one live beam: the rest comes from the next beams, which have
    the lowest score there is, one of them ended."""
    groups, width, vocab, eos = 5, 6, 4003, 77
    z = logits(3, groups, width, vocab, dtype)
    z[:, 0, 3:] = -INF
    z[1, 1, 6:] = z[2, 1] = -INF
    z[3, 1:] = torch.finfo(dtype).min
    s = torch.full((groups, width), LOWEST, device="cuda")
    s[:, 0] = -3.0
    s[4] = LOWEST
    last = torch.zeros(groups, width, dtype=torch.int32, device="cuda")
    last[:, 2] = eos
    for k in (2, 3, 6, 16, 64):
        check(z, s, k, last, eos)


@TYPES
def test_equal_logits_of_zero(dtype):
    """Nothing to tell apart at all."""
    z = torch.zeros(3, 5, 30001, device="cuda", dtype=dtype)
    z[1, :, ::2] = -INF
    for k in (1, 9, 64):
        check(z, torch.zeros(3, 5, device="cuda"), k)


def test_in_place_with_ties():
    """Scores and last tokens are replaced while ties are settled."""
    groups, width, vocab, eos = 4, 8, 5003, 9
    z = logits(4, groups, width, vocab)
    s = torch.full((groups, width), 1e30, device="cuda")
    last = torch.zeros(groups, width, dtype=torch.int32, device="cuda")
    last[:, 0] = last[1, 1] = last[2, :7] = eos
    last[3] = eos
    before = s.clone(), last.clone()
    parents = torch.empty_like(last)
    sv.spec_beam_select(z, s, parents, last, s, last_tokens=last, eos_token=eos)
    check(z, before[0], width, before[1], eos, got=(parents, last, s))
    assert [t.tolist() for t in run(z, *before[:1], width, before[1], eos)] == [t.tolist() for t in (parents, last, s)]


@TYPES
@pytest.mark.parametrize("groups,width,vocab,k", [(6, 24, 31, 5), (3, 64, 2000, 28), (4, 42, 15001, 40), (40, 6, 1300, 6),
                                                  (17, 12, 50001, 9)])
def test_beams_that_are_sure(groups, width, vocab, k, dtype):
    """One token has all the probability, in beams of equal scores, some of which have ended: the
    logarithm of such a sum is zero."""
    z = logits(vocab, groups, width, vocab, dtype, std=300.0)
    best = z.float().amax(-1, keepdim=True)
    z = torch.where(z.float() < best - 40.0, z, z.float().amin().to(dtype))      # no second one near the best
    z.scatter_(2, torch.randint(vocab, (groups, width, 1), device="cuda", generator=torch.Generator("cuda").manual_seed(1)),
               best.to(dtype))
    s = torch.full((groups, width), -1.5, device="cuda")
    s[:, ::3] = 0.0
    last = torch.zeros(groups, width, dtype=torch.int32, device="cuda")
    last[:, 4::5] = vocab - 1
    check(z, s, k, last, vocab - 1)
    check(z, s, k)


@TYPES
@pytest.mark.parametrize("groups,width,vocab,k", [(6, 24, 64, 5), (3, 64, 2000, 28), (4, 42, 15001, 40), (40, 6, 1300, 6)])
def test_beams_of_equally_many_tokens(groups, width, vocab, k, dtype):
    """A row's tokens are equally likely, the same number of them in several beams, others masked:
    sums of ones."""
    gen = torch.Generator("cuda").manual_seed(vocab)
    order = torch.rand(groups, width, vocab, device="cuda", generator=gen).argsort(-1)
    some = torch.randint(1, 4, (groups, width, 1), device="cuda", generator=gen) * (vocab // 4)
    level = torch.randint(-3, 4, (groups, width, 1), device="cuda", generator=gen).float()
    z = torch.where(order < some, level, -INF).to(dtype)
    check(z, torch.zeros(groups, width, device="cuda"), k)


@TYPES
def test_logits_that_are_logarithms_of_probabilities(dtype):
    """The best of them are zeros, below which there are floats that fp64 scores do not tell from
    zero; the k-th best is another."""
    z = torch.log_softmax(logits(5, 20, 6, 5003, std=8.0), -1)
    z[::2, :, 7] = 0.0
    z[1::3, ::2] = torch.where(z[1::3, ::2] < z[1::3, ::2].amax(-1, keepdim=True), -80.0, 0.0)
    for k in (1, 6, 20):
        check(z.to(dtype), torch.zeros(20, 6, device="cuda"), k)


@TYPES
@pytest.mark.parametrize("k", [1, 8, 30, 64])
def test_few_tokens_far_into_the_rows(dtype, k):
    """Beams that offer some tokens each, anywhere in long rows, at one score."""
    groups, width, vocab = 6, 9, 30011
    z = logits(8, groups, width, vocab, dtype)
    keep = torch.rand(z.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(2)) < 5 / vocab
    keep[:, ::4, -1] = keep[1, :, 4095:4098] = keep[2, 1, 511:514] = True
    keep[3, 2:] = False
    z = torch.where(keep, z, torch.full_like(z, -INF))
    check(z, torch.full((groups, width), -1e30, device="cuda"), k)
