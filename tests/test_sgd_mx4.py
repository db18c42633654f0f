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


def test_gradients_and_aggregation_take_separate_seeds(monkeypatch, capsys):
    """Every seed that the command's layer and its aggregators are given: none twice
    within one, none of both."""
    rounded, aggregated = [], []

    class Layer:
        def __init__(self, tokens, inputs, outputs, device):
            self.shape = tokens, inputs

        def load(self, w):
            pass

        def forward(self, x):
            return torch.zeros(self.shape[0], 1)

        def backward(self, dy, seed):
            rounded.append(seed)
            return None, torch.zeros(1, self.shape[1])

    def aggregator(*a):
        def run(grads, d, seed):
            aggregated.append(seed)
            return grads[:, :d].mean(0)
        return run

    make_problem = sgd.make_problem
    monkeypatch.setattr(sgd, "Mx4Linear", Layer)
    monkeypatch.setattr(sgd, "QuantisedAggregate", aggregator)
    monkeypatch.setattr(sgd, "Mx4Aggregate", aggregator)
    monkeypatch.setattr(sgd, "make_problem", lambda n, M, rows, seed, device: make_problem(n=n, M=M, rows=rows, seed=seed))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    T, M, seeds, settings = 5, 2, 3, len(sgd.CONFIGS) + 1
    monkeypatch.setattr("sys.argv", ["sgd", "--n", "8", "--M", str(M), "--rows", "16", "--T", str(T), "--gradients", "mx4"])
    assert sgd.main() == 0
    assert len(rounded) == settings * seeds * 2 * T * M and len(set(rounded)) == len(rounded)
    assert len(aggregated) == (settings - 1) * seeds * 2 * T and len(set(aggregated)) == seeds * T
    assert not set(rounded) & set(aggregated)
    assert all(0 <= s < 1 << 64 for s in rounded + aggregated)
    del rounded[:]
    p = make_problem(n=8, M=M, rows=16, seed=1)
    sgd.Mx4Gradients(p)(p, torch.zeros(8, dtype=torch.float64), torch.zeros(M, 8))
    assert min(rounded) >= sgd.GRADIENT_SEEDS > max(aggregated)
