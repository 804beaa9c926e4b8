"""packing_report without a GPU: measurements replaced by given costs."""
import sys

import numpy as np
import pytest

from paper_2503_17924_amd import binding as B
from paper_2503_17924_amd import packing_report as R
from paper_2503_17924_amd import profile_kernels as PK


def run(monkeypatch, capsys, *args):
    """-> (the linear cost that each packer was made with, the printed text); attention costs 3 ps per token^2, the ends 200000 ps per token"""
    costs = []

    class Packer(B.Packer):
        def __init__(self, n_microbatch, l_max, cost_a, cost_b, *more):
            costs.append(cost_b)
            super().__init__(n_microbatch, l_max, cost_a, cost_b, *more)

    monkeypatch.setattr(B, "Packer", Packer)
    monkeypatch.setattr(PK, "time_rank", lambda torch, binding, q, cu, *a, **k: float((np.diff(cu).astype(np.float64) ** 2).sum()) * 3e-9)
    monkeypatch.setattr(R, "time_vocabulary", lambda torch, binding, docs, *a, **k: sum(docs) * 200000e-9)
    monkeypatch.setattr(sys, "argv", ["packing_report", "--iterations", "4", *args])
    R.main()
    return costs, capsys.readouterr().out


def test_packers_balance_the_linear_cost_that_the_step_counts(monkeypatch, capsys):
    costs, text = run(monkeypatch, capsys, "--vocab", "1000")
    assert costs == [R.COST_B + 200000] * 2
    assert "200000 ps per token" in text


def test_without_a_vocabulary_the_packers_keep_their_cost(monkeypatch, capsys):
    costs, text = run(monkeypatch, capsys)
    assert costs == [R.COST_B] * 2 and "lookup" not in text


def test_least_squares_of_a_linear_cost():
    assert R.per_token_ps([1000, 3000], [2e-6 * 1000, 2e-6 * 3000]) == pytest.approx(2000)
    assert R.per_token_ps([1, 2], [1e-9, 4e-9]) == pytest.approx(9 / 5)
