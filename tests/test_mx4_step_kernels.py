"""The library holds the step's kernels that calls can launch, and no others."""
import re

from paper_2109_12497_amd import LIB_PATH


def chosen(M, d):
    """The kernel's rows and whether outputs and gradients pass the caches by, as launched."""
    if 4 * d <= 46 << 20 and (M >= 5 or d <= 1 << 18):
        return "spread"
    rows = 2 if M <= 2 else 4 if M <= 4 else 8 if M <= 8 else 16
    return rows, 4 * d > 46 << 20, 4 * d > 46 << 20 and 4 * d * M > 256 << 20


def test_every_step_kernel_can_be_launched():
    edges = [1, 1 << 18, 46 << 18] + [(256 << 18) // M for M in range(1, 17)] + [1 << 30]
    reached = {chosen(M, d + e) for M in range(1, 17) for d in edges for e in (0, 1)}
    blob = open(LIB_PATH, "rb").read()
    built = {(int(r), nt == b"1", loads == b"1") for r, nt, loads in
             re.findall(rb"k_mx4_stepILi(\d+)ELb([01])ELb([01])EE", blob)}
    assert built == reached - {"spread"}
