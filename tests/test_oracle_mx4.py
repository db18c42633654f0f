"""The 64-bit implementation of microscaled 4-bit floating point, pinned: its
uniform words to the C oracle's, its scale rule and rounding to exact rational
arithmetic, its stochastic rounding to the mean it must have."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import mx4


def test_words_are_the_oracles(orc):
    w = mx4.words(3, 43, 5, 0x123456789ABCDEF0)
    for row in range(3):
        for col in (0, 1, 7, 8, 21, 42):
            assert int(w[row, col]) == orc.uniform_word(0x123456789ABCDEF0, 5 + row, col)


@pytest.mark.parametrize("top", [0.0, 2.0 ** -149, 2.0 ** -126, 6 * 2.0 ** -126, 6.0000005 * 2.0 ** -126, 0.3, 5.9999995,
                                 6.0, 6.0000005, 7.9, 8.0, 11.999999, 12.0, 12.000001, 3.4028235e38])
def test_scale_rule(top):
    top = float(np.float32(top))
    b = int(mx4.bytes_of(np.array([[top]]))[0, 0])
    e = b - 127
    assert 1 <= b <= 253 and Fraction(top) <= 6 * Fraction(2) ** e
    assert e == -126 or Fraction(top) > 6 * Fraction(2) ** (e - 1)


def test_scale_of_what_is_not_finite():
    assert mx4.bytes_of(np.array([[np.inf, np.nan, 1.0]])).tolist() == [[255, 255, 125]]
    x = np.zeros((1, 40), dtype=np.float32)
    x[0, 3], x[0, 35] = np.nan, -2.0
    codes, b = mx4.quantize(x, None)
    assert b.tolist() == [[255, 126]] and not codes[0, :16].any()
    v = mx4.decode(codes, b, 40)
    assert np.isnan(v[0, :32]).all() and v[0, 35] == -2.0 and not v[0, 36:].any()


def test_nearest_by_fractions():
    """Every multiple of 1/64 up to 6: the nearest level, ties to the even code."""
    y = np.arange(0, 385) / 64.0
    x = np.zeros((1, 32), dtype=np.float32)
    for v in y:
        x[0, 0], x[0, 1] = v, 6.0  # 6 holds the scale at 1
        f = mx4.fields(x, mx4.bytes_of(mx4.block_max(x)), None)
        best = min(range(8), key=lambda c: (abs(Fraction(float(mx4.LEVELS[c])) - Fraction(float(v))), c & 1))
        assert f[0, 0] == best


def test_stochastic_is_unbiased_exactly():
    """Over every value of the uniform word the mean code is the element to
    within 2^-32 of a step: counted by the threshold that the words meet."""
    for y in (0.1, 0.5, 1.2, 1.99, 2.5, 3.75, 5.0, 5.9):
        x = np.zeros((1, 32), dtype=np.float32)
        x[0, 0], x[0, 1] = y, 6.0
        b = mx4.bytes_of(mx4.block_max(x))
        exact = Fraction(float(x[0, 0]))
        lo = max(c for c in range(8) if mx4.LEVELS[c] <= float(x[0, 0]))
        low, high = Fraction(float(mx4.LEVELS[lo])), Fraction(float(mx4.LEVELS[min(lo + 1, 7)]))
        first, last = 0, 2 ** 32  # bisect the number of words that round up
        while first < last:
            mid = (first + last) // 2
            r = np.full((1, 32), mid, dtype=np.uint64)
            if mx4.fields(x, b, r)[0, 0] == lo + 1:
                first = mid + 1
            else:
                last = mid
        mean = low + (high - low) * Fraction(first, 2 ** 32)
        assert 0 <= exact - mean < (high - low) * Fraction(1, 2 ** 32)


def test_aggregate_of_equal_rows_on_the_grid():
    """Rows that lie on the grid come back exactly whatever the words."""
    x = np.tile(np.array([[0, 0.5, -1, 1.5, 2, -3, 4, 6] * 5], dtype=np.float32) * 0.25, (3, 1))
    b, s, out = mx4.aggregate(x, 40, 7)
    assert (b == 125).all() and np.array_equal(s, (x[0] * 4 * 2 * 3).astype(np.int64))
    # 1 / 3 rounds by at most 2^-24 of itself, the product once more
    assert np.all(np.abs(out - x[0]) <= 2 * 2.0 ** -24 * np.abs(x[0]))
