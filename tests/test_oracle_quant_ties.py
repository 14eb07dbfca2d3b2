"""Pins of the 8-bit oracle next to the border of two codes: rational arithmetic, for every value."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import quant


def rational(rows):
    """Codes of rows of Fractions: rint(127 u / max|u|), ties to even (Python's round of a Fraction)."""
    tops = [max(abs(v) for v in row) for row in rows]
    return [[round(127 * u / m) for u in row] for row, m in zip(rows, tops)]


@pytest.mark.parametrize("e", [20, 33, 39, 40, 41, 42, 45, 50])
def test_values_past_a_tie_take_their_own_code(e):
    d = 2.0 ** -e
    for sign in (1, -1):
        assert quant.codes(sign * np.array([[127.0, 0.5 + d, 2.5 + d]]), exact=True)[0].tolist() == [[sign * 127, sign, 3 * sign]]
        assert quant.codes(sign * np.array([[127.0, 1.5 - d, 3.5 - d]]), exact=True)[0].tolist() == [[sign * 127, sign, 3 * sign]]
    assert quant.codes(np.array([[127.0, 0.5, 1.5, 2.5]]), exact=True)[0].tolist() == [[127, 0, 2, 2]]


def test_sums_and_products_in_rational_arithmetic():
    r = np.random.default_rng(5)
    M, D = 30, 60
    x = (r.integers(0, 127, (M, D)) + 0.5) * r.choice([-1, 1], (M, D))
    y = np.exp2(-r.integers(20, 46, (M, D)).astype(np.float64)) * r.choice([-1, 0, 1], (M, D))
    x[:, 7], y[:, 7] = 127, 0
    rows = [[Fraction(a) + Fraction(b) for a, b in zip(u, v)] for u, v in zip(x.tolist(), y.tolist())]
    assert quant.codes(x + y, exact=True)[0].tolist() == rational(rows)
    # products with gamma (24 bits each; the norm's factor divides out)
    s, g = r.integers(1, 1 << 24, (M, D)).astype(np.float64), r.integers(1, 1 << 24, D).astype(np.float64)
    rows = [[Fraction(a) * Fraction(b) for a, b in zip(u, g.tolist())] for u in s.tolist()]
    assert quant.rms(s, g, 1e-6)[0].tolist() == rational(rows)


def test_a_layer_norms_ties_are_ties():
    # differences from the mean of half of the largest, gamma one, beta zero: 63.5, to the even code;
    # the norm's own roundings would take it to either side
    for f in (1.0, 3.0, 0.1, 1e-3):
        s = np.array([[2.0, -2.0, 1.0, -1.0, 0.0, 0.0, 0.0]]) * f
        assert quant.layer(s, np.ones(7), np.zeros(7), 1e-6)[0].tolist() == [[127, -127, 64, -64, 0, 0, 0]]
