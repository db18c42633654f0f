"""The 64-bit implementation's mean of the step on microscaled 4-bit codes,
pinned to exact rational arithmetic: one rounding to binary32."""
from fractions import Fraction

import numpy as np

from oracle import mx4


def nearest32(x: Fraction) -> np.float32:
    """The binary32 number next to x, ties to even."""
    at = np.float32(float(x))
    near = [np.nextafter(at, np.float32(-np.inf)), at, np.nextafter(at, np.float32(np.inf))]
    return min((v for v in near if np.isfinite(v)),
               key=lambda v: (abs(Fraction(float(v)) - x), int(v.view(np.int32)) & 1))


def test_mean_is_rounded_once():
    rng = np.random.default_rng(1)
    for M in (1, 2, 3, 5, 7, 12, 100, 1001, 3_000_001, 178_956_970):
        total = np.concatenate([rng.integers(-12 * M, 12 * M + 1, size=56), [0, 1, -1, M, -M, 5 * M, 12 * M, -12 * M]])
        for byte in (1, 2, 24, 100, 127, 200, 252):
            out = mx4.mean(total, np.full(2, byte, dtype=np.uint8), M)
            want = [nearest32(Fraction(int(t), M) * Fraction(2) ** (byte - 128)) for t in total]
            assert np.array_equal(out.view(np.int32) & 0x7FFFFFFF, np.array(want).view(np.int32) & 0x7FFFFFFF)
            assert (np.sign(out) == np.sign(np.array(want))).all()


def test_mean_of_the_extreme_bytes():
    assert np.isnan(mx4.mean(np.array([5, 0]), np.array([255], dtype=np.uint8), 3)).all()
    assert mx4.mean(np.array([36, -35]), np.array([253], dtype=np.uint8), 3).tolist() == [np.inf, -np.inf]
    assert mx4.mean(np.array([3, 1]), np.array([0], dtype=np.uint8), 3)[0] == 2.0 ** -127  # 0 is read as 1
