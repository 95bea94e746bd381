"""GPU parity of the products with 4-bit weights against the float64 oracle
(oracle.drafting).

What a packed matrix stands for is compared exactly.

A product is compared element-wise with a bound made of its roundings.  A weight has
two significant bits and an x eight, so each product w x is exact in fp32; the sum of
K of them in any order, each addition off by at most 2^-23 of its result (a rounding
to nearest is off by half of that; the matrix cores may cut bits off), is off by at
most (K + 16) 2^-23 A, A = sum |w x|; 16 more terms for the joins of waves and splits.
Products below 2^-126 may be flushed, K 2^-126 in all.  A bf16 output adds half a step,
2^-8 of the output.  gate_up: with dg, du the bounds of its sums, silu has a slope of at
most 1.1, so 1.1 dg |u| + |silu(g)| du + 1.1 dg du; e^-g in fp32 is off by its
argument's rounding, (|g| + 8) 2^-21 of silu(g) with the quotient's own, and where e^-g
overflows (g < -87) silu is below 1e-35.
"""

import numpy as np
import pytest
import torch

import paper_2512_04752_amd as sv
from oracle import drafting as O

pytestmark = pytest.mark.gpu


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)


def numbers(seed, *shape, std=1.0):
    rng = np.random.default_rng(seed)
    x = rng.normal(0, std, shape) * np.exp(0.6 * rng.normal(size=shape[-1]))
    return bf16(x)


def unpacked(m):
    return m.unpack().double().cpu().numpy()


# ---- pack and unpack ---------------------------------------------------------

@pytest.mark.parametrize("rows,cols", [(1, 32), (16, 128), (17, 160), (5, 96), (40, 512), (33, 544), (130, 2080)])
def test_pack_holds_the_nearest_numbers(rows, cols):
    w = numbers(rows + cols, rows, cols, std=0.02)
    m = sv.W4Matrix(w.cuda())
    assert np.array_equal(unpacked(m), O.quantise(w.double().numpy()))


def test_pack_edges():
    """Zeros and negative zeros, midpoints, both ends of the exponents, infinities and NaN."""
    w = torch.zeros(10, 64, dtype=torch.bfloat16)
    w[1, :32] = -0.0
    mid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    w[2, :8], w[2, 8:16] = mid, -mid
    w[3, :8], w[3, 31] = mid * 2.0 ** -40, 6 * 2.0 ** -40
    w[4, 0], w[4, 1] = 2.0 ** -126, 1.5 * 2.0 ** -120
    w[5, 0], w[5, 33] = 3.0e38, -3.3e38
    w[6, 0] = 2.0 ** -133
    w[7, 3], w[7, 40] = float("inf"), 1.0
    w[8, 63], w[8, 0] = float("nan"), 2.0
    w[9, 5] = -float("inf")
    got = sv.W4Matrix(w.cuda()).unpack().cpu()
    want = O.quantise(w.double().numpy())
    assert np.array_equal(np.isnan(got.double().numpy()), np.isnan(want))
    keep = ~np.isnan(want)
    assert np.array_equal(got.double().numpy()[keep], want[keep])
    assert not (torch.signbit(got) & (got == 0)).any()


def test_pack_strided_rows_and_bytes_outside():
    big = numbers(3, 50, 416, std=0.1).cuda()
    w = big[:, 96:96 + 288]
    n = sv.spec_w4_bytes(50, 288)
    data = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    sv.spec_w4_pack(w, data[:n])
    out = torch.full((50, 416), 7.0, dtype=torch.bfloat16, device="cuda")
    sv.spec_w4_unpack(data[:n], out[:, 64:64 + 288])
    assert (data[n:] == 0xA5).all()
    assert (out[:, :64] == 7).all() and (out[:, 352:] == 7).all()
    assert np.array_equal(out[:, 64:352].double().cpu().numpy(), O.quantise(w.double().cpu().numpy()))


# ---- products ----------------------------------------------------------------

def sum_bound(K, A):
    return (K + 16) * 2.0 ** -23 * A + K * 2.0 ** -126


def check(got, want, bound):
    got = got.double().cpu().numpy()
    bad = np.nonzero(~(np.abs(got - want) <= bound))
    assert len(bad[0]) == 0, f"{len(bad[0])} of {got.size} outside, first at {[int(b[0]) for b in bad]}: " \
                             f"{got[bad][0]} not {want[bad][0]} within {bound[bad][0]}"


ROWS = [1, 2, 15, 16, 17, 32, 33, 63, 64, 65, 100, 128, 129, 200, 256, 257, 300, 513]
SHAPES = [(1, 32), (16, 128), (293, 96), (77, 640), (256, 256), (512, 1024), (1040, 288)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_linear(shape):
    rows, cols = shape
    m = sv.W4Matrix(numbers(1, rows, cols, std=0.02).cuda())
    w = unpacked(m)
    for n in ROWS:
        x = numbers(n, n, cols)
        want, A = O.linear(x.double().numpy(), w)
        bound = sum_bound(cols, A)
        xc = x.cuda()
        out = torch.full((n, rows), 9.0, dtype=torch.float32, device="cuda")
        sv.spec_w4_linear(m, xc, out)
        check(out, want, bound)
        half = torch.full((n, rows), 9.0, dtype=torch.bfloat16, device="cuda")
        sv.spec_w4_linear(m, xc, half)
        check(half, want, bound + 2.0 ** -8 * np.abs(want) + 2.0 ** -8 * bound)


@pytest.mark.parametrize("rows,cols", [(2048, 2048), (4096, 14336), (14336, 4096), (20000, 1088)])
@pytest.mark.parametrize("n", [1, 4, 16, 24, 64, 96, 700])
def test_linear_large(rows, cols, n):
    """Model sizes: sums and outputs computed on the GPU in float64."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    w = torch.empty(rows, cols, device="cuda").normal_(0, 0.02, generator=gen).to(torch.bfloat16)
    x = torch.empty(n, cols, device="cuda").normal_(0, 1, generator=gen).to(torch.bfloat16)
    m = sv.W4Matrix(w)
    held = m.unpack().double().T.contiguous()
    want, A = x.double() @ held, x.double().abs() @ held.abs()
    out = torch.empty(n, rows, device="cuda")
    sv.spec_w4_linear(m, x, out)
    check(out, want.cpu().numpy(), sum_bound(cols, A.cpu().numpy()))


def test_linear_adds():
    rows, cols = 300, 512
    m = sv.W4Matrix(numbers(1, rows, cols, std=0.02).cuda())
    for n in (1, 33, 130):
        x = numbers(n, n, cols)
        base = torch.from_numpy(np.random.default_rng(n).normal(size=(n, rows)).astype(np.float32)).cuda()
        out = base.clone()
        sv.spec_w4_linear(m, x.cuda(), out, add=True)
        want, A = O.linear(x.double().numpy(), unpacked(m))
        want = want + base.double().cpu().numpy()
        check(out, want, sum_bound(cols, A) * 1.01 + 2.0 ** -24 * np.abs(want))


@pytest.mark.parametrize("n", [1, 16, 40, 64, 100, 260])
@pytest.mark.parametrize("shape", [(16, 32), (293, 160), (512, 1024), (1056, 576)], ids=str)
def test_gate_up(shape, n):
    rows, cols = shape
    gate, up = (sv.W4Matrix(numbers(i, rows, cols, std=0.05).cuda()) for i in (1, 2))
    x = numbers(n, n, cols)
    out = torch.full((n, rows), 9.0, dtype=torch.bfloat16, device="cuda")
    sv.spec_w4_gate_up(gate, up, x.cuda(), out)
    g, Ag = O.linear(x.double().numpy(), unpacked(gate))
    u, Au = O.linear(x.double().numpy(), unpacked(up))
    dg, du, s = sum_bound(cols, Ag), sum_bound(cols, Au), O.silu(g)
    want = s * u
    bound = 1.1 * dg * np.abs(u) + np.abs(s) * du + 1.1 * dg * du + (np.abs(g) + 8) * 2.0 ** -21 * np.abs(want) \
        + 1e-35 * np.abs(u)
    check(out, want, bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want))


@pytest.mark.parametrize("rows,cols,n", [(40, 70016, 16), (17, 70016, 1), (24, 300000, 16), (5, 131072, 3), (33, 64, 5000),
                                         (64, 4096, 4097)])
def test_long_and_tall(rows, cols, n):
    """Columns that take many pieces of LDS, or more than it has; rows in the thousands."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    m = sv.W4Matrix(torch.empty(rows, cols, device="cuda").normal_(0, 0.02, generator=gen).bfloat16())
    x = torch.empty(n, cols, device="cuda").normal_(0, 1, generator=gen).bfloat16()
    held = m.unpack().double().T.contiguous()
    want, A = x.double() @ held, x.double().abs() @ held.abs()
    out = torch.empty(n, rows, device="cuda")
    sv.spec_w4_linear(m, x, out)
    check(out, want.cpu().numpy(), sum_bound(cols, A.cpu().numpy()))


@pytest.mark.parametrize("n", [3, 40])
def test_rows_gigabytes_apart(n):
    """The last token's state of long samples: one row of every 128 MB."""
    rows, cols = 96, 256
    m = sv.W4Matrix(numbers(1, rows, cols, std=0.02).cuda())
    big = torch.empty(n, 1 << 26, dtype=torch.bfloat16, device="cuda")
    x = big[:, 4096:4096 + cols]
    x.copy_(numbers(n, n, cols))
    out = torch.empty(n, rows, device="cuda")
    sv.spec_w4_linear(m, x, out)
    want, A = O.linear(x.double().cpu().numpy(), unpacked(m))
    check(out, want, sum_bound(cols, A))


@pytest.mark.parametrize("n", [1, 20, 70, 300])
def test_strided_and_unaligned(n):
    """Rows of a fused projection's output in, columns of a wider buffer out, at odd places."""
    rows, cols = 151, 160
    m = sv.W4Matrix(numbers(1, rows, cols, std=0.02).cuda())
    big = numbers(n, n, 400).cuda()
    x = big[:, 88:88 + cols]
    want, A = O.linear(x.double().cpu().numpy(), unpacked(m))
    for dtype in (torch.float32, torch.bfloat16):
        buf = torch.full((n, 401), 3.0, dtype=dtype, device="cuda")
        sv.spec_w4_linear(m, x, buf[:, 7:7 + rows])
        bound = sum_bound(cols, A)
        check(buf[:, 7:7 + rows], want, bound if dtype == torch.float32 else
              bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want))
        assert (buf[:, :7] == 3).all() and (buf[:, 7 + rows:] == 3).all()


@pytest.mark.parametrize("n", [3, 18, 50, 90, 280])
def test_a_row_that_is_not_finite_stays_alone(n):
    rows, cols = 200, 256
    m = sv.W4Matrix(numbers(1, rows, cols, std=0.02).cuda())
    x = numbers(n, n, cols).cuda()
    clean, out = (torch.empty(n, rows, device="cuda") for _ in range(2))
    sv.spec_w4_linear(m, x, clean)
    bad = n // 2
    x[bad, 5], x[bad, 200] = float("inf"), float("nan")
    sv.spec_w4_linear(m, x, out)
    keep = [i for i in range(n) if i != bad]
    assert torch.equal(out[keep], clean[keep]) and torch.isnan(out[bad]).all()


def test_weights_that_are_not_finite():
    """A group without a scale makes NaN of its own outputs only."""
    w = numbers(1, 40, 256, std=0.02)
    w[3, 100] = float("nan")
    m = sv.W4Matrix(w.cuda())
    for n in (1, 40, 150):
        out = torch.empty(n, 40, device="cuda")
        sv.spec_w4_linear(m, numbers(n, n, 256).cuda(), out)
        assert torch.isnan(out[:, 3]).all() and torch.isfinite(out[:, [i for i in range(40) if i != 3]]).all()


@pytest.mark.parametrize("n", [1, 16, 48, 200])
def test_same_bits_each_time_and_on_replay(n):
    """Eager, on another stream and replayed from a graph; an overwritten workspace is no matter."""
    rows, cols = 1024, 4096
    m = sv.W4Matrix(numbers(1, rows, cols, std=0.02).cuda())
    gate = sv.W4Matrix(numbers(2, rows, cols, std=0.02).cuda())
    x = numbers(n, n, cols).cuda()
    ws = torch.full((max(1, sv.spec_w4_workspace_bytes(rows, cols, n)),), 0xFF, dtype=torch.uint8, device="cuda")

    def both(a, b):
        sv.spec_w4_linear(m, x, a, workspace=ws)
        sv.spec_w4_gate_up(gate, m, x, b, workspace=ws)

    want = torch.empty(n, rows, device="cuda"), torch.empty(n, rows, dtype=torch.bfloat16, device="cuda")
    both(*want)
    got = [torch.zeros_like(t) for t in want]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sv.spec_w4_linear(m, x, got[0], stream=side)
    sv.spec_w4_gate_up(gate, m, x, got[1], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(*got)
    for step in range(3):
        for t in got:
            t.fill_(5)
        ws.fill_(step)
        x.copy_(numbers(n + step, n, cols))
        both(*want)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_no_rows():
    m = sv.W4Matrix(numbers(1, 16, 32).cuda())
    out = torch.empty(0, 16, device="cuda")
    sv.spec_w4_linear(m, torch.empty(0, 32, dtype=torch.bfloat16, device="cuda"), out)
    sv.spec_w4_gate_up(m, m, torch.empty(0, 32, dtype=torch.bfloat16, device="cuda"), out.to(torch.bfloat16))
    torch.cuda.synchronize()


def test_refusals_of_tensors():
    m = sv.W4Matrix(numbers(1, 48, 64).cuda())
    x, out = numbers(2, 4, 64).cuda(), torch.empty(4, 48, device="cuda")
    for bad in (dict(x=x.float()), dict(x=x[:, :32]), dict(x=x.cpu()), dict(x=x.T.contiguous().T),
                dict(out=out[:3]), dict(out=out[:, :40]), dict(out=out.double()), dict(out=out.cpu()),
                dict(out=out.to(torch.bfloat16), add=True),
                dict(workspace=torch.empty(256, device="cuda"))):
        with pytest.raises(ValueError):
            sv.spec_w4_linear(**{**dict(m=m, x=x, out=out), **bad})
    with pytest.raises(sv.SpecError, match="16-byte"):
        sv.spec_w4_linear(m, torch.empty(4 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(4, 64), out)
    with pytest.raises(sv.SpecError, match="stride"):
        sv.spec_w4_linear(m, torch.empty(4, 65, dtype=torch.bfloat16, device="cuda")[:, :64], out)
    other = sv.W4Matrix(numbers(1, 32, 64).cuda())
    with pytest.raises(sv.SpecError, match="gate is"):
        sv.spec_w4_gate_up(m, other, x, out.to(torch.bfloat16))
    for w in (numbers(1, 4, 40).cuda(), numbers(1, 4, 64), torch.empty(4, 64, device="cuda")):
        with pytest.raises((ValueError, sv.SpecError)):
            sv.W4Matrix(w)
