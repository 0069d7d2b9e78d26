"""Implicit feedback on the table: GET, softmax loss or distillation, INC, CLOCK together."""
import numpy as np
import pytest
import torch

from gen import workload

pytestmark = pytest.mark.gpu


def _step(X, N, users, q, eta):
    """X after one worker's step in fp64: rows of the batch's users, then of all items."""
    L, R = X[users], X[N:]
    s = L @ R.T
    p = np.exp(s - s.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    g = p - q
    out = np.zeros_like(X)
    np.add.at(out, users, -eta * (g @ R))
    out[N:] -= eta * (g.T @ L)
    return out


@pytest.mark.parametrize("s", [0, 2])
def test_clocks_of_the_loss_follow_the_formula(s):
    """Three clocks of two workers against fp64 steps from the read versions.  An update
    sums at most 300 fp32 terms of at most eta, so 1e-5 (1 + |x|) holds it."""
    from paper_1410_8043_gb300.implicit import Trainer

    N, M, K, P, B, eta = 60, 300, 12, 2, 40, 0.1
    tr = Trainer(N, M, K, P, s, B)
    X = [tr.table.read_table(0).double().cpu().numpy()]
    rng = np.random.default_rng(3)
    for c in range(1, 4):
        v, clk = tr.table.read_schedule()
        assert clk == c
        new = X[-1].copy()
        for p in range(P):
            users, picks = rng.integers(0, N, B), rng.integers(0, M, B)
            tr.learn(p, torch.as_tensor(users, dtype=torch.int32, device="cuda"),
                     torch.as_tensor(picks, dtype=torch.int32, device="cuda"), eta)
            new += _step(X[v[p]], N, users, np.eye(M)[picks], eta)
        tr.table.clock()
        X.append(new)
        got = tr.table.read_table(c).double().cpu().numpy()
        assert (np.abs(got - new) <= 1e-5 * (1 + np.abs(new))).all()
    assert np.abs(X[-1] - X[0]).max() > 1e-2
    tr.close()


def test_command_trains_and_distills():
    """The command's run on the tiny workload: both models learn (the loss starts at
    log 1000 = 6.9, the divergence of lists of 20 from near log(1000 / 20))."""
    from paper_1410_8043_gb300.implicit import run

    rows = []
    run(workload("tiny"), 40, 512, 0.2, 8, 0.05, 20, 10, rows.append)
    loss = [r["loss"] for r in rows if "loss" in r]
    div = [r["divergence"] for r in rows if "divergence" in r]
    assert len(loss) == 5 and len(div) == 5
    assert 6.8 < loss[0] < 7.0 and loss[-1] < loss[0] - 0.3
    assert div[-1] < div[0] - 0.1
