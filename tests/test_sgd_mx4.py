"""The convergence demo on microscaled 4-bit codes, with the 64-bit
implementation as the aggregator: the variance and the bound that it states for
exact gradients, and that it states none for others."""
import numpy as np
import pytest
import torch

from oracle import mx4
from paper_2109_12497_amd import sgd


@pytest.fixture(scope="module")
def problem():
    return sgd.make_problem(n=96, M=4, rows=200, seed=1)


def aggregate(scales):
    assert scales == sgd.MX4
    return lambda grads, d, seed: torch.from_numpy(mx4.aggregate(grads.numpy(), d, seed)[2])


def test_variance_stays_under_its_bound(problem):
    """The mean square distance of the aggregate from the exact mean, at the
    start and near the solution, where blocks' widths differ most."""
    p = problem
    agg, n = aggregate(sgd.MX4), 40
    for theta in (torch.zeros(p.n, dtype=torch.float64), 0.99 * p.theta_star):
        g = torch.zeros((p.M, p.n), dtype=torch.float32)
        sgd.shard_gradients(p, theta, g)
        want = g.double().mean(0)
        off = [float(((agg(g, p.n, seed).double() - want) ** 2).sum()) for seed in range(n)]
        assert 0.0 < np.mean(off) <= sgd.variance_bound(p, sgd.MX4)


def test_table_with_exact_gradients(problem):
    row = sgd.convergence_table(problem, aggregate, T=60, seeds=(0, 1), configs={"mx4": sgd.MX4})["mx4"]
    assert row["sigma2_bound"] == sgd.variance_bound(problem, sgd.MX4)
    assert -1e-9 <= row["gap_avg"] <= row["bound"]


def test_no_bound_for_other_gradients(problem):
    """Gradients that are not the exact ones are outside the theorems."""
    def biased(p, theta, out):
        sgd.shard_gradients(p, theta, out)
        out += 1.0

    for configs, make in (({"mx4": sgd.MX4}, aggregate), ({"fp32 mean": None}, lambda scales: sgd.mean_aggregate)):
        (row,) = sgd.convergence_table(problem, make, T=3, seeds=(0,), configs=configs, gradients=biased).values()
        assert "bound" not in row and "sigma2_bound" not in row
        assert all(np.isfinite(v) for v in row.values()) and set(row) >= {"eta", "gap_avg", "gap_tail_fixed_step"}
