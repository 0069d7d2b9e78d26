"""Lookup, layer norm, softmax and AdamW together: the model that trains by itself."""
import math

import pytest
import torch

from gen import workload

pytestmark = pytest.mark.gpu


def _loss64(tables, weight, bias, tied, inputs, picks, scale, row_weight):
    """The sum of weighted losses, from fp64 leaves."""
    items, rows = tables[0], tables[0 if tied else 1]
    kept = inputs >= 0
    x = torch.where(kept[:, None], rows[inputs.long().clamp(min=0)] * scale, 0.0)
    d = x - x.mean(1, keepdim=True)
    h = d / (d.square().mean(1, keepdim=True) + 1e-5).sqrt() * weight + bias
    s = h @ items.T
    loss = torch.logsumexp(s, 1) - s.gather(1, picks.long().clamp(min=0)[:, None])[:, 0]
    return (torch.where(picks >= 0, loss, 0.0) * row_weight).sum()


def _batch(n, N, M, tied, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    inputs = torch.randint(0, M if tied else N, (n,), generator=g, device="cuda", dtype=torch.int32)
    picks = torch.randint(0, M, (n,), generator=g, device="cuda", dtype=torch.int32)
    inputs[::7], picks[::5] = -1, -1
    return inputs, picks, torch.rand(n, generator=g, device="cuda") + 0.5


# A gradient is a sum of at most n = 70 rows' terms (items: 70 of p h, inputs 70) below 10 each; fp32 sums, softmax
# probabilities (1e-5, as in the softmax's tests) and the norm's 140 eps keep it within 5e-5 of 1 + what it is; 16-bit rows
# round h, p and dh: each off by half a unit of a term, 2^-8 (bf16) or 2^-11 (fp16) of ten terms' size at most.
TOL = {torch.float32: 5e-5, torch.bfloat16: 10 * 2.0**-8, torch.float16: 10 * 2.0**-11}


@pytest.mark.parametrize("dtype", list(TOL))
@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("n, N, M, K", [(1, 5, 9, 8), (70, 40, 300, 24), (70, 400, 1000, 100), (64, 30, 50, 33)])
def test_gradients_follow_autograd(n, N, M, K, tied, dtype):
    from paper_1410_8043_gb300.implicit import DenseTrainer

    m = DenseTrainer(None if tied else N, M, K, n, dtype=dtype, scale=math.sqrt(K), init=1 / math.sqrt(K))
    inputs, picks, row_weight = _batch(n, N, M, tied, n + M)
    if n == 1:
        inputs[0], picks[0] = 3, 4
    _, grads = m.gradients(inputs, picks, row_weight)
    leaves = [t.double().requires_grad_() for t in ([m.items] if tied else [m.items, m.inputs]) + [m.weight, m.bias]]
    _loss64(leaves[:-2], leaves[-2], leaves[-1], tied, inputs, picks, math.sqrt(K), row_weight.double()).backward()
    for got, leaf in zip(grads, leaves):
        err = (got.double() - leaf.grad).abs()
        assert bool((err <= TOL[dtype] * (1 + leaf.grad.abs())).all()), float((err / (1 + leaf.grad.abs())).max())
    m.close()


@pytest.mark.parametrize("tied", [False, True])
def test_steps_follow_the_formula(tied):
    """Four steps against fp64.  A gradient off by 1e-4 moves a step lr m / (sqrt(v) + eps) by 2 lr 1e-4 / eps at most:
    4 steps of lr = 1e-2, eps = 1e-2: 1e-3, of movements of 4e-2."""
    from paper_1410_8043_gb300.implicit import DenseTrainer

    N, M, K, n, lr, eps, decay = 60, 200, 20, 50, 1e-2, 1e-2, 0.1
    m = DenseTrainer(None if tied else N, M, K, n, eps=eps, weight_decay=decay)
    p = [t.double().clone() for t in m.params]
    start = [t.clone() for t in p]
    first, second = [torch.zeros_like(t) for t in p], [torch.zeros_like(t) for t in p]
    for t in range(1, 5):
        inputs, picks, row_weight = _batch(n, N, M, tied, t)
        m.learn(inputs, picks, lr, weight=row_weight)
        leaves = [x.clone().requires_grad_() for x in p]
        _loss64(leaves[:-2], leaves[-2], leaves[-1], tied, inputs, picks, 1.0, row_weight.double()).backward()
        for k, leaf in enumerate(leaves):
            first[k] = 0.9 * first[k] + 0.1 * leaf.grad
            second[k] = 0.999 * second[k] + 0.001 * leaf.grad**2
            step = lr * (first[k] / (1 - 0.9**t)) / ((second[k] / (1 - 0.999**t)).sqrt() + eps)
            p[k] = p[k] * (1 - lr * (decay if k < len(p) - 2 else 0.0)) - step
    for got, want, before in zip(m.params, p, start):
        assert float((got.double() - want).abs().max()) <= 1e-3
        assert float((want - before).abs().max()) > 1e-2
    m.close()


@pytest.mark.parametrize("dtype, bits", [(torch.float32, 32), (torch.bfloat16, 8)])
def test_a_captured_step(dtype, bits):
    """A whole step in a CUDA graph, replayed on batches that change, gives the bits of the steps made by hand."""
    from paper_1410_8043_gb300.implicit import DenseTrainer

    N, M, K, n = 300, 500, 32, 200
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        one = DenseTrainer(N, M, K, n, dtype=dtype, state_bits=bits)
    two = DenseTrainer(N, M, K, n, dtype=dtype, state_bits=bits)
    torch.cuda.synchronize()
    inputs, picks, _ = _batch(n, N, M, False, 0)
    a, b, lr = inputs.clone(), picks.clone(), torch.tensor(1e-2, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        loss = one.learn(a, b, lr)
    for t in range(1, 4):
        inputs, picks, _ = _batch(n, N, M, False, t)
        a.copy_(inputs), b.copy_(picks)
        graph.replay()
        by_hand = two.learn(inputs, picks, lr)
        assert torch.equal(loss, by_hand)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(one.params, two.params)) and torch.equal(one.items, two.items)
    del graph
    one.close(), two.close()


def test_a_model_of_popular_items_over_many_tokens():
    """Batches that take the sort: 30000 tokens, tied, against autograd in fp64 (sums of 30000 terms of |p| |h| <= 5:
    the popular row's are off by 1e-6 of their mass)."""
    from paper_1410_8043_gb300.implicit import DenseTrainer

    M, K, n = 400, 64, 30_000
    m = DenseTrainer(None, M, K, n, init=1 / math.sqrt(K))
    g = torch.Generator("cuda").manual_seed(1)
    inputs = (torch.rand(n, generator=g, device="cuda") ** 4 * M).int()
    picks = (torch.rand(n, generator=g, device="cuda") ** 4 * M).int()
    weight = torch.full((n,), 1 / n, device="cuda")
    _, grads = m.gradients(inputs, picks, weight)
    leaves = [t.double().requires_grad_() for t in m.params]
    _loss64(leaves[:-2], leaves[-2], leaves[-1], True, inputs, picks, 1.0, weight.double()).backward()
    for got, leaf in zip(grads, leaves):
        assert float((got.double() - leaf.grad).abs().max()) <= 1e-5 * (1 + float(leaf.grad.abs().max()))
    m.close()


@pytest.mark.parametrize("dtype, bits", [(torch.float32, 32), (torch.bfloat16, 8)])
def test_command_runs(dtype, bits):
    from paper_1410_8043_gb300.implicit import run_dense

    rows = []
    run_dense(workload("tiny"), 12, 256, 0.01, bits, dtype, 5, rows.append)
    assert [r["step"] for r in rows] == [1, 5, 10, 12] and all(math.isfinite(r["loss"]) for r in rows)
