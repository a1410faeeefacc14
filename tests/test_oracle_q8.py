"""The oracle of rows in 8 bits against closed forms and its own definition."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import q8_oracle as Q


def test_cut16():
    for x in (Fraction(1), Fraction(1, 3), Fraction(65535), Fraction(65537), Fraction(2 ** 40 + 1), Fraction(1, 2 ** 140)):
        c = Q.cut16(x)
        assert c <= x < c * (1 + Fraction(1, 2 ** 15))
        while c.denominator > 1:
            c *= 2
        n = c.numerator
        while n % 2 == 0:
            n //= 2
        assert n < 2 ** 16
    assert Q.cut16(Fraction(65537)) == 65536 and Q.cut16(Fraction(2 ** 17 + 1)) == 2 ** 17


def test_whole_numbers_are_kept():
    h = np.array([[127.0, -126, 1, 0, -127], [254, 2, -4, 0, 6]])
    q, s = Q.quantize(h, "signed")
    assert s.tolist() == [1.0, 2.0] and np.array_equal(q * s[:, None], h)
    h = np.array([[255.0, 0, -3, 17]])
    q, s = Q.quantize(h, "relu")
    assert s[0] == 1.0 and q.tolist() == [[255, 0, 0, 17]]


def test_ties_and_small_values():
    q, s = Q.quantize([[127.0, 0.5, 1.5, -2.5, 0.4999]], "signed")
    assert q.tolist() == [[127, 0, 2, -2, 0]]
    q, s = Q.quantize([[255.0, 0.5, 1.5, 1e-30, -1e-30]], "relu")
    assert q.tolist() == [[255, 1, 2, 1, 0]]


@pytest.mark.parametrize("kind", ["signed", "relu"])
def test_error_within_half_a_step(kind):
    rng = np.random.default_rng(3)
    h = rng.standard_normal((50, 33)) * np.exp(rng.normal(0, 20, (50, 1)))
    q, s = Q.quantize(h, kind)
    back = q * s[:, None]
    t = h if kind == "signed" else np.maximum(h, 0)
    # at the top: levels * s is up to 2^-15 below the largest value; relu's least code is 1
    step = 0.5 + 255 * 2.0 ** -15 if kind == "signed" else 1.0
    assert np.all(np.abs(back - t) <= step * s[:, None])
    assert np.array_equal(q > 0, h > 0) or kind == "signed"


def test_rows_without_numbers():
    q, s = Q.quantize([[0.0, 0], [np.nan, 1], [np.inf, 1], [-5, -np.inf]], "relu")
    assert s[0] == 2.0 ** -126 and np.isnan(s[1:]).all() and not q.any()


def test_product_and_gradients_by_hand():
    s = Q.product([[2, -3]], np.array([0.5]), [[1, 4], [0, -1]], np.array([2.0, 1.0]))
    assert s.tolist() == [[-10.0, 1.5]]
    h, w, g = np.array([[1.0, 0], [2, 3]]), np.array([[1.0], [-2]]), np.array([[4.0], [5]])
    dw, dz, db = Q.transform_bwd(h, w, g, h > 0, 0.5)
    assert dw.tolist() == [[14.0], [15.0]]
    assert dz.tolist() == [[8.0, 0], [10, -20]] and db.tolist() == [18.0, -20]
