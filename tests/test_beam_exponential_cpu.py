"""The exponential of the beams' normalisers, on the CPU with the constants that the kernel's
source has: 2^f on |f| <= 1/2 by a polynomial, and e^d where the result's exponent is a
normal one."""

import os
import re

import numpy as np

from paper_2512_04752_amd import build

SOURCE = open(os.path.join(build.CSRC, "beam_search.hip")).read()
C = [float(x) for x in re.search(r": c\{([^}]*)\}", SOURCE).group(1).split(",")]
LOG2E, BIG = 1.44269504088896340736, 6755399441055744.0 + 4096.0


def polynomial(f):
    y = np.full_like(f, C[7])
    for c in C[6::-1]:
        y = y * f + c
    return y


def exponential(d):
    """The kernel's steps, products and sums rounded once each (it fuses them)."""
    d = np.asarray(d, np.float64)
    m = d * LOG2E + BIG
    f = (d.astype(np.longdouble) * np.longdouble(LOG2E) + (BIG - m)).astype(np.float64)
    n = m.view(np.int64) & 0xffffffff
    y = polynomial(f).view(np.int64)
    hi = (y >> 32) + (n << 20) & 0xffffffff
    return ((hi << 32) | (y & 0xffffffff)).astype(np.uint64).view(np.float64)


def test_constants_are_those_of_the_source():
    assert len(C) == 8 and "log2e = 1.44269504088896340736;" in SOURCE and "6755399441055744.0 + 4096.0" in SOURCE


def test_polynomial():
    """Largest relative error 4.67e-11: of degree 7 and with a 1 at 0 that is the smallest."""
    f = np.linspace(-0.5, 0.5, 200001)
    off = np.abs(polynomial(f) / np.exp2(f.astype(np.longdouble)) - 1).max()
    assert 4.6e-11 < off < 4.7e-11
    assert polynomial(np.zeros(1))[0] == 1


def test_exponential_over_its_range():
    """d log2 e is off by 2^-53 of up to 1022, and f as much: 2e-13 more."""
    d = np.concatenate((np.linspace(-708, 690, 400001), [-708.0, -690.0, -600.0, -0.0, 0.0, 1e-300, 600.0, 690.0]))
    want = np.exp(d.astype(np.longdouble))
    assert (np.abs(exponential(d) / want - 1) < 5e-11).all()
    assert (exponential([0.0, -0.0]) == 1).all()
