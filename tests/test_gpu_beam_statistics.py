"""The choice of beams where a row's pieces carry their statistics over several steps of a
wave: numbers that are not finite, wherever they stand, and logits of any size.

The reference takes log softmax(z)[y] as (z_y - max z) - log sum exp(z - max z) in float64,
which is exact to 1e-13 for logits of any size (the difference of two fp32 numbers is
exact while they are within 2^29 of each other, and counts for nothing beyond).  Parents and
tokens are equal, scores within 1e-9 and half a step of fp32."""

import numpy as np
import pytest
import torch

import paper_2512_04752_amd as sv
from tests.test_gpu_beam import logits, scores

pytestmark = pytest.mark.gpu
INF = float("inf")


def reference(z, s, k):
    z, s = z.double(), s.double()
    groups = z.shape[0]
    top = z.amax(-1, keepdim=True)                         # a NaN when there is one
    key = s[..., None] + ((z - top) - torch.log(torch.exp(z - top).sum(-1, keepdim=True)))
    key = torch.where((top.abs() < INF) & (s.abs() < INF)[..., None], key, -INF).view(groups, -1)
    got, at = torch.sort(key, dim=1, descending=True, stable=True)
    got, at = got[:, :k], at[:, :k]
    none = got == -INF
    return (torch.where(none, -1, at // z.shape[2]), torch.where(none, -1, at % z.shape[2]), got)


def check(z, s, k, off=1e-9):
    groups = z.shape[0]
    parents, tokens = (torch.full((groups, k), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    new = torch.full((groups, k), 7.0, device="cuda")
    sv.spec_beam_select(z, s, parents, tokens, new)
    want = reference(z, s, k)
    assert parents.tolist() == want[0].tolist()
    assert tokens.tolist() == want[1].tolist()
    some = want[2] > -INF
    assert torch.equal(new > -INF, some)
    assert ((new.double() - want[2]).abs() <= off + 2.0 ** -24 * want[2].abs())[some].all()


# many rows, so that a wave goes through its segment in several batches, the last of them partial
GROUPS, WIDTH, VOCAB = 17, 12, 50001


@pytest.fixture(params=[torch.float32, torch.bfloat16], ids=str)
def rows(request):
    return logits(1, GROUPS, WIDTH, VOCAB, request.param), scores(1, GROUPS, WIDTH)


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("k", [4, 24])
def test_nan_in_every_piece_of_a_row(rows, k, seed):
    """A NaN takes its beam out, at tokens spread over the segments' batches and lanes; the last
    batch of the last segment has no numbers for some lanes."""
    z, s = rows
    rng = np.random.default_rng(seed)
    n = GROUPS * WIDTH
    at = np.concatenate((VOCAB - 1 - rng.integers(0, 2600, size=n // 2), rng.integers(0, VOCAB, size=n - n // 2)))
    at = rng.permutation(at).reshape(GROUPS, WIDTH)
    for g in range(GROUPS):
        for w in range(WIDTH):
            if w != g % WIDTH:
                z[g, w, int(at[g, w])] = float("nan")
    check(z, s, k)


@pytest.mark.parametrize("what", [float("nan"), INF], ids=str)
@pytest.mark.parametrize("k", [4, 24])
def test_not_finite_before_masked_tokens(rows, k, what):
    """All that follows is masked, or all but what another batch, lane or segment has."""
    z, s = rows
    for g in range(GROUPS):
        for w in range(WIDTH - 1):
            at = (g * WIDTH + w) * 233 % (VOCAB - 8)
            z[g, w, at] = what
            z[g, w, at + 1:(VOCAB, at + 3000, VOCAB - 2)[w % 3]] = -INF
    check(z, s, k)


def patterns(n):
    """Rows of small whole numbers: up and down once, with every batch of a wave, every token."""
    at = torch.arange(n, device="cuda")
    batch, half = at // 1024, (at >= n // 2).long()
    return torch.stack((half, -half, batch % 2, -(batch % 2), batch % 3 - 1, at % 2, batch // 2 % 2 + at % 2, at % 7 - 3))


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("k", [4, 24])
def test_steps_at_large_magnitudes(sign, k):
    """Near 2^e neighbouring floats are 2^(e - 23) apart: below, around and beyond what an
    exponential holds.  A normaliser of 2^e rounded to fp64 is off by 2^(e - 53), and its
    difference by as much."""
    steps = patterns(100003)
    sizes = torch.tensor([2.0 ** e for e in range(22, 42)], dtype=torch.float64, device="cuda")[:, None, None]
    exact = sign * sizes * 1.5 + steps * sizes * 2.0 ** -23
    z = exact.float()
    assert torch.equal(z.double(), exact)
    check(z, scores(3, *z.shape[:2]), k, off=1e-9 + 2 * sizes[..., 0] * 2.0 ** -53)


@pytest.mark.parametrize("k", [4, 24])
def test_steps_around_what_an_exponential_holds(k):
    """Rises and falls around 32, and by 590 .. 720, where terms begin and cease to count."""
    sizes = [1.0, 20.0, 31.0, 31.999, 32.0, 33.0, 36.0, 64.0, 590.0, 599.5, 600.0, 600.5, 610.0, 679.5, 680.0, 680.5,
             689.0, 690.0, 691.0, 700.0, 709.0, 720.0]
    z = patterns(100003) * torch.tensor(sizes, device="cuda")[:, None, None]
    z += torch.linspace(0, 1, z.shape[2], device="cuda")
    check(z, scores(3, *z.shape[:2]), k)


def test_the_most_rows_there_can_be():
    """2^22 rows in segments for teams of waves; few of them have a token that is not masked."""
    groups, width, vocab, k = 65536, 64, 8000, 16
    z = torch.full((groups, width, vocab), -INF, dtype=torch.bfloat16, device="cuda")
    picked = [0, 1, 40000, groups - 1]
    z[picked] = logits(5, len(picked), width, vocab, torch.bfloat16)
    s = scores(5, groups, width)
    parents, tokens = (torch.full((groups, k), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    new = torch.full((groups, k), 7.0, device="cuda")
    sv.spec_beam_select(z, s, parents, tokens, new)
    want = reference(z[picked], s[picked], k)
    assert torch.equal(parents[picked].long(), want[0]) and torch.equal(tokens[picked].long(), want[1])
    parents[picked] = -1
    assert (parents == -1).all()
    del z
    torch.cuda.empty_cache()


BOUND = 4 * 4.7e-11 + 1e-12


def check_normaliser(z, rows):
    """Scores that are nearly nothing, an fp32 number less the best candidate's logarithm: fp32
    rounds 1e-6 by 2^-24 of it, and what is left is the normaliser's error.  A term is the
    product of at most four exponentials (its own to its lane's reference, once from there to a
    later one, to its wave's and to its row's; a second later reference would be 32 above it),
    each off by at most 4.7e-11 of itself, and so are a sum and its logarithm by four times that;
    the doubles' roundings are below 1e-12."""
    groups = len(z)
    near = torch.log_softmax(z[rows].double(), -1).amax(-1)
    s = torch.zeros(groups, 1, device="cuda")
    s[rows] = (-near).float()
    parents, tokens = (torch.empty(groups, 4, dtype=torch.int32, device="cuda") for _ in range(2))
    new = torch.empty(groups, 4, device="cuda")
    sv.spec_beam_select(z, s, parents, tokens, new)
    best = (s[rows].double() + near)[:, 0]
    assert (best.abs() < 1e-6).all()
    assert ((new[rows, 0].double() - best).abs() <= BOUND + 2.0 ** -24 * best.abs()).all()


def test_slow_rises_beside_steep_ones():
    """One lane's logits rise by 700 at every step of a wave, far below the others', which rise a
    little each time."""
    groups, vocab = 4096, 128000             # one segment a row, 125 steps of 1024
    at = torch.arange(vocab, device="cuda")
    z = (at // 1024 * 0.001)[None, None].repeat(groups, 1, 1)
    z[:, :, at % 256 < 4] = -100000.0        # 16 of a step's 1024 are a lane's
    z[:, :, at % 1024 == 0] += at[at % 1024 == 0] // 1024 * 700.0
    rows = [0, 1, 2000, groups - 1]
    z[rows] += (at % 256 >= 4) * 1e-4 * torch.rand(len(rows), 1, vocab, device="cuda",
                                                    generator=torch.Generator("cuda").manual_seed(1))
    check_normaliser(z, rows)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("groups,vocab", [(6, 1), (6, 64), (6, 1000), (6, 50001), (6, 128256), (300, 50001), (4096, 9001)])
@pytest.mark.parametrize("std", [0.01, 0.5, 5.0])
def test_normalisers_to_their_bound(groups, vocab, dtype, std):
    check_normaliser(logits(vocab, groups, 1, vocab, dtype, std=std), [0, 1, groups // 2, groups - 1])
