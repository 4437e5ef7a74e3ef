"""Rotary frequencies and tables against their formulas, written out (no GPU)."""
import math

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
