"""Two stochastic roundings in a row, the second of a value formed from the
first: without bias with words of their own, biased where they share them."""
from fractions import Fraction

import numpy as np

from oracle import mx4


def element(x, top, word):
    """What x stands for after rounding with `word` in a block whose largest is `top`."""
    block = np.zeros((1, 32), dtype=np.float32)
    block[0, 0], block[0, 1] = x, top
    b = mx4.bytes_of(mx4.block_max(block))
    f = mx4.fields(block, b, np.full((1, 32), word, dtype=np.uint64))
    return mx4.decode(mx4.pack(f), b, 32)[0, 0]


def test_a_chain_needs_two_words():
    """1.25 (a quarter of the way between 1 and 1.5 and so on: all thresholds
    are multiples of 2^-6) rounded, multiplied by 1.5 and rounded on a coarser
    scale, over words in the middles of 64 equal parts: the means are exact."""
    x, n = 1.25, 64
    words = [(2 * i + 1) << 25 for i in range(n)]
    first = [element(x, 6.0, w) for w in words]
    second = {v: [element(1.5 * v, 9.0, w) for w in words] for v in set(first)}
    own = sum(Fraction(v) for a in first for v in second[a]) / n ** 2
    shared = sum(Fraction(second[a][i]) for i, a in enumerate(first)) / n
    assert own == Fraction(3, 2) * Fraction(x)
    assert shared != own
