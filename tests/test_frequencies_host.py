"""CPU tests of the rotation's frequencies: angles as turns in 64-bit fractions, exact to the last bit wherever they are taken."""
import random
from fractions import Fraction

import pytest

import paper_2305_13450_amd as ds


def two_pi():
    """To 2^-600: pi = 16 atan(1/5) - 4 atan(1/239)."""
    one = 1 << 640
    def atan_of_inverse(n):
        s, term, k = 0, one // n, 1
        while term:
            s += term // k if k % 4 == 1 else -(term // k)
            term, k = term // (n * n), k + 2
        return s
    return Fraction(2 * (16 * atan_of_inverse(5) - 4 * atan_of_inverse(239)), one)


def test_large_angles_are_exact_or_refused():
    turn, r = two_pi(), random.Random(5)
    for e in list(range(-40, 100, 7)) + [99]:
        for _ in range(4):
            x = r.choice((-1, 1)) * r.uniform(0.5, 1.0) * 2.0 ** e
            assert ds.rope_frequencies([x]).item() % 2 ** 64 == round(Fraction(x) / turn * 2 ** 64) % 2 ** 64, x
    for x in (2.0 ** 100, -(2.0 ** 100), 1e60, 1.7e308):
        with pytest.raises(ValueError):
            ds.rope_frequencies([0.5, x])
