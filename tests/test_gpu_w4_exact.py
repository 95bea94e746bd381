"""Products with 4-bit weights whose every partial sum is a number of fp32: x of -1, 0 and 1,
weights that are codes at one scale.  A sum of up to 349525 halves of at most 12 stays
below 2^22 halves in any order, so outputs are equal to the exact ones, and a column
that is left out, or taken twice, shows at any length."""

import pytest
import torch

import paper_2512_04752_amd as sv

pytestmark = pytest.mark.gpu

# columns that take many pieces of LDS, or more than it has (few rows), and split tiles (more)
LONG = [(40, 70016, 16), (17, 70016, 1), (24, 300000, 16), (24, 300000, 1), (5, 131072, 3), (5, 131072, 16), (33, 64, 5000),
        (64, 4096, 4097), (40, 70016, 17), (24, 300000, 40), (5, 131072, 200), (2048, 2048, 1), (4096, 14336, 16),
        (4096, 14336, 24), (4096, 14336, 64), (4096, 14336, 300), (14336, 4096, 4), (20000, 1088, 96), (2048, 8192, 128)]


def codes(gen, rows, cols):
    """Numbers that a matrix in 4 bits holds as they are: a group's largest is 4 or 6, so that its scale is 1."""
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device="cuda")
    w = grid[torch.randint(8, (rows, cols), generator=gen, device="cuda")]
    first = torch.randint(32, (rows, cols // 32, 1), generator=gen, device="cuda")
    w.view(rows, -1, 32).scatter_(2, first, 6.0)
    w *= torch.randint(2, w.shape, generator=gen, device="cuda") * 2 - 1
    return w.bfloat16()


def matrix(w):
    m = sv.W4Matrix(w)
    assert torch.equal(m.unpack(), w)
    return m


def product(x, w):
    """Exact: whole numbers of halves below 2^53, in pieces of columns."""
    out = torch.zeros(len(x), len(w), dtype=torch.float64, device="cuda")
    for a, b in zip(x.split(8192, 1), w.split(8192, 1)):
        out += a.double() @ b.double().T.contiguous()
    return out


@pytest.mark.parametrize("rows,cols,n", LONG)
def test_linear(rows, cols, n):
    gen = torch.Generator(device="cuda").manual_seed(rows + n)
    w = codes(gen, rows, cols)
    m = matrix(w)
    x = (torch.randint(3, (n, cols), generator=gen, device="cuda") - 1).bfloat16()
    want = product(x, w)
    out = torch.full((n, rows), 9.0, device="cuda")
    sv.spec_w4_linear(m, x, out)
    assert torch.equal(out.double(), want)
    sv.spec_w4_linear(m, x, out, add=True)
    assert torch.equal(out.double(), 2 * want)
    half = torch.full((n, rows), 9.0, dtype=torch.bfloat16, device="cuda")
    sv.spec_w4_linear(m, x, half)
    assert torch.equal(half, want.float().bfloat16())


@pytest.mark.parametrize("rows,cols,n", LONG)
def test_gate_up(rows, cols, n):
    """A gate of 32 or more is its own silu in fp32.  It comes from one group of a row, which
    walks over the columns; the rows of x are 1, 2 or 4 all along."""
    gen = torch.Generator(device="cuda").manual_seed(cols + n)
    w = codes(gen, rows, cols)
    gate = torch.zeros(rows, cols // 32, 32, dtype=torch.bfloat16, device="cuda")
    row = torch.arange(rows, device="cuda")
    gate[row, row * 7919 % (cols // 32), :8] = 4.0
    x = (2.0 ** (torch.arange(n, device="cuda") % 3))[:, None].expand(n, cols).bfloat16()
    scale = x[:, :1].double()
    out = torch.full((n, rows), 9.0, dtype=torch.bfloat16, device="cuda")
    sv.spec_w4_gate_up(matrix(gate.view(rows, cols)), matrix(w), x, out)
    assert torch.equal(out, (32 * scale * scale * w.double().sum(1)).float().bfloat16())
