"""Trainer on a stream that is not the caller's: inputs that the caller's stream still
makes, results that it uses at once, memory that it hands on."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _softmax(s):
    e = np.exp(s - s.max(1, keepdims=True))
    return e / e.sum(1, keepdims=True)


@pytest.mark.parametrize("kind", ["loss", "distill"])
@pytest.mark.parametrize("built_on,used_on", [("side", "current"), ("current", "side"), ("side", "other")])
def test_calls_from_another_stream(kind, built_on, used_on):
    """Three clocks against fp64 steps from the version read (one worker, no staleness).  An
    update sums at most 100 fp32 terms of at most eta: 1e-5 (1 + |x|) holds it.  Lists name
    each row's whole teacher softmax over four items."""
    from paper_1410_8043_gb300.implicit import Trainer

    N, M, K, B, eta = 80, 500, 16, 64, 0.1
    streams = {"current": torch.cuda.current_stream(), "side": torch.cuda.Stream(), "other": torch.cuda.Stream()}
    tr = Trainer(N, M, K, 1, 0, B, max_top=4, stream=streams[built_on])
    table = tr.table
    rng = np.random.default_rng(5)
    torch.cuda.synchronize()
    with torch.cuda.stream(table.stream):
        X = table.read_table(0).double().cpu().numpy()
    for c in range(1, 4):
        users, ids = rng.permutation(N)[:B], np.stack([rng.permutation(M)[:4] for _ in range(B)])
        z = rng.standard_normal((B, 4)).astype(np.float32)
        with torch.cuda.stream(streams[used_on]):
            made = [torch.as_tensor(x, device="cuda") for x in (users.astype(np.int32), ids.astype(np.int32), z)]
            given = [torch.zeros_like(x) for x in made]
            torch.cuda.current_stream().synchronize()
            torch.cuda._sleep(20_000_000)  # what follows on this stream comes late
            for x, y in zip(given, made):
                x.copy_(y)
            h, w = tr.rows(0, given[0])
            seen = (h.double(), w.double())
            if kind == "loss":
                loss = tr.learn(0, given[0], given[1][:, 0].contiguous(), eta)
            else:
                loss = tr.learn_from(0, given[0], given[1], given[2], eta)
            total = loss.double() * 1.0
            for x in (h, w, loss, *given):  # (late work of this stream on memory that it gives back)
                x.zero_()
            del h, w, loss, given
            table.clock()
            total, seen = total.cpu().numpy(), [x.cpu().numpy() for x in seen]
        L, R = X[users], X[N:]
        p, q = _softmax(L @ R.T), np.zeros((B, M))
        if kind == "loss":
            q[np.arange(B), ids[:, 0]] = 1.0
            want = -np.log((p * q).sum(1))
        else:
            np.put_along_axis(q, ids, _softmax(z.astype(np.float64)), 1)
            want = (q * (np.log(np.where(q > 0, q, 1.0)) - np.log(p))).sum(1)
        assert np.abs(seen[0] - L).max() < 1e-5 and np.abs(seen[1] - R).max() < 1e-5
        assert np.abs(total - want).max() < 1e-4
        X = X.copy()
        dL, dR = (p - q) @ R, (p - q).T @ L
        X[users] -= eta * dL
        X[N:] -= eta * dR
        torch.cuda.synchronize()
        with torch.cuda.stream(table.stream):
            got = table.read_table(c).double().cpu().numpy()
        assert (np.abs(got - X) <= 1e-5 * (1 + np.abs(X))).all()
    tr.close()
