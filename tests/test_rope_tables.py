"""Rotary frequencies and tables against their formulas, written out (no GPU)."""
import math
from fractions import Fraction

import numpy as np
import pytest

import paper_2606_24467_gb300 as ckv


def ramp(rot_dim, base, factor, length, low, high):
    """Frequencies whose share that stays falls linearly in the pair's number
    between the pairs whose waves make `high` and `low` turns over `length`, rounded
    outwards, the one at least 0 and the other at most rot_dim - 1."""
    def number(turns):
        return rot_dim * math.log(length / (2 * math.pi * turns)) / (2 * math.log(base))

    first = max(math.floor(number(high)), 0)
    last = min(math.ceil(number(low)), rot_dim - 1)
    i = np.arange(rot_dim // 2)
    f = float(base) ** (-2.0 * i / rot_dim)
    keep = 1 - np.clip((i - first) / (last - first), 0.0, 1.0)
    return f * keep + f / factor * (1 - keep)


@pytest.mark.parametrize("rot_dim, base, factor, length, low, high", [
    (128, 10000.0, 4.0, 4096.0, 1.0, 32.0),
    (128, 10000.0, 4.0, 32768.0, 1.0, 32.0),
    (128, 10000.0, 4.0, 65536.0, 1.0, 32.0),     # from here on `low` turns lie past the last pair
    (128, 10000.0, 4.0, 131072.0, 1.0, 32.0),
    (64, 10000.0, 4.0, 131072.0, 1.0, 32.0),
    (128, 10000.0, 8.0, 8192.0, 0.1, 32.0),
    (128, 500000.0, 16.0, 1048576.0, 1.0, 32.0),
    (96, 10000.0, 40.0, 4096.0, 1e-6, 1.0),      # past rot_dim - 1, too
    (20, 1000.0, 2.0, 777.0, 0.5, 4.0),
])
def test_ramp_by_its_formula(rot_dim, base, factor, length, low, high):
    got = ckv.rope_frequencies(rot_dim, base, "ramp", factor, length, low, high)
    # (logarithms and powers of two libraries: some units in the last place of exponents up to 14)
    np.testing.assert_allclose(got, ramp(rot_dim, base, factor, length, low, high), rtol=1e-13)


def turns_exactly(f):
    """f / 2 pi modulo 1 in units of 2^-64, as a rational (pi by Machin's formula)."""
    bits = 400

    def atan_of_inverse(x):
        term = total = (1 << bits) // x
        for n in range(3, bits, 2):
            term //= -x * x
            total += term // n
        return total

    two_pi = 8 * (4 * atan_of_inverse(5) - atan_of_inverse(239))
    return Fraction(f) * (1 << bits) * (1 << 64) / two_pi % (1 << 64)


@pytest.mark.parametrize("frequencies", [
    [1.0, -1.0, 100.0, -100.0, 1048575.7, -1048575.7, 2.0 ** 20, 0.0],
    [1e-6, -1e-6, 1e-17, -1e-17, 2 * math.pi, -2 * math.pi, 1e-300, -5e-324],
    [3.0 ** -i for i in range(16, 24)],
    list(500000.0 ** (-np.arange(64) / 64.0)),
])
def test_tables_hold_turns(frequencies):
    rope = ckv.Rope(2 * len(frequencies), frequencies=np.array(frequencies))
    for f, t in zip(frequencies, rope.struct.turns):
        gap = abs(int(t) - turns_exactly(f))
        # a quotient of doubles, 2 pi rounded: 1.5 * 2^-53 of it, at most |f| 2^-55 (1.5 < 2 pi / 4); and cut to units
        bound = abs(Fraction(f)) / 4 * Fraction(1, 1 << 53) * (1 << 64) + 1
        assert min(gap, (1 << 64) - gap) <= bound, (f, float(gap), float(bound))
