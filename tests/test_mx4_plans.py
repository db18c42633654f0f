"""The workspace of the microscaled product over the whole range of sizes: the
choice of a form runs on the host alone."""
import itertools

import pytest

import paper_2109_12497_amd as uq

SIZES = [-1, 0, 1, 15, 16, 17, 64, 65, 128, 129, 1000, 2 ** 16 + 1, 2 ** 24, 2 ** 31 - 1, 2 ** 31, 2 ** 62]


@pytest.mark.parametrize("k", SIZES)
def test_every_size_has_a_workspace(k):
    for m, n in itertools.product(SIZES, SIZES):
        size = uq.uq_mx4_matmul_workspace_bytes(m, n, k)
        # at most 8 parts of 2^24 outputs, rows padded to four columns
        assert 256 <= size <= 8 * 4 * 4 * 2 ** 24 + 256
        assert size % 256 == 0
