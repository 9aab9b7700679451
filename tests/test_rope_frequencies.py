"""Frequencies of the rotary positions (commfuse_rope_make, host only) against the formulas in 60 decimal digits.

A frequency is kept in turns per position as a 64-bit binary fraction.  Bounds, in units of 2^-64 relative to the frequency:
  power, quotient by 2 pi and the fraction in extended precision (64 bits)      8, and one unit of the fraction
  r in 64-bit floating point: off by at most 2^-52 (w + 1), w = (n + low) / (high - low) <= (high + low) / (high - low) for the ramp over
  turns and 1 for the one over the index, which moves f (r + (1 - r) / factor) by (1 - 1 / factor) f at most that, and that is (factor - 1)
  times as much relatively, since the frequency is at least f / factor."""
import math
from decimal import Decimal, getcontext
from fractions import Fraction

import pytest

from paper_2604_24013_amd import binding as cf

getcontext().prec = 60
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import os
    if not os.path.exists(cf.LIB_PATH):
        from paper_2604_24013_amd import build
        build.build()
    cf.load()


def turns(j, rot, base, scaling, factor, trained, low, high):
    base, factor, trained, low, high = (Decimal(x) for x in (base, factor, trained, low, high))
    f = (base.ln() * (Decimal(-2 * j) / rot)).exp()
    r = Decimal(0)
    if scaling == "wavelength":
        r = (trained * f / (2 * PI) - low) / (high - low)
    elif scaling == "index":
        at = lambda t: rot * (trained / (2 * PI * t)).ln() / (2 * base.ln())
        first, last = max(0, math.floor(at(high))), min(rot - 1, math.ceil(at(low)))
        r = 1 - (j - first) / max(Decimal(last - first), Decimal("0.001"))
    r = min(Decimal(1), max(Decimal(0), r))
    return f * (r + (1 - r) / factor) / (2 * PI)


def check(rot, base, scaling, factor, trained, low, high):
    made = cf.rope_make(256, rot, "half", base=base, scaling=scaling, factor=factor, trained_len=trained, low=low, high=high)
    width = (high + low) / (high - low) if scaling == "wavelength" else 1.0
    units = 8 + (0 if scaling == "linear" else (factor - 1) * (width + 1) * 2 ** 12)
    for j in range(rot // 2):
        want = Fraction(turns(j, rot, base, scaling, factor, trained, low, high))
        assert abs(Fraction(made.turn[j], 2 ** 64) - want) <= want * Fraction(units) / 2 ** 64 + Fraction(1, 2 ** 64), (j, float(want), made.turn[j] / 2 ** 64)


@pytest.mark.parametrize("rot", [2, 32, 64, 96, 128, 256])
@pytest.mark.parametrize("base, trained, low, high", [(1e4, 131072, 1.0, 32.0), (1e4, 65536, 0.5, 4.0), (100.0, 4096, 1.0, 32.0), (5e5, 2 ** 22, 1.0, 8.0)])
def test_ramp_over_the_index_may_end_behind_the_last_pair(rot, base, trained, low, high):
    """Where even the slowest pair makes more than `low` turns over the trained length, the ramp goes on beyond the last pair (up to index
    rot_dim - 1): pairs are between trained and stretched as far as their own turns say."""
    check(rot, base, "index", 4.0, trained, low, high)


@pytest.mark.parametrize("rot", [2, 24, 64, 96, 128, 256])
@pytest.mark.parametrize("base, scaling, factor, trained, low, high", [
    (1e4, "linear", 1.0, 0, 1.0, 4.0), (1e4, "linear", 2.5, 0, 1.0, 4.0), (1.5, "linear", 1.0, 0, 1.0, 4.0), (1e18, "linear", 1e9, 0, 1.0, 4.0),
    (5e5, "wavelength", 8.0, 8192, 1.0, 4.0), (1e4, "wavelength", 2.0, 4096, 0.25, 16.0), (1e6, "index", 4.0, 32768, 1.0, 32.0),
    (1e4, "index", 40.0, 4096, 1.0, 32.0), (2.0, "index", 2.0, 7, 1.0, 1.1)])
def test_frequencies_in_sixty_digits(rot, base, scaling, factor, trained, low, high):
    check(rot, base, scaling, factor, trained, low, high)
