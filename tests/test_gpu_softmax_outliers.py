"""One row of H, or some items of W, far larger than the rest: everything that does not
depend on them has to come out as if they were not there (GPU, fp32 rows).

The reference is the definition in fp64 on the rows and items that are left when the
outliers, the rows that score them, and those rows' targets are taken out; their share of
what is compared is below 1e-30.  Tolerances, with eps = 2^-24: a score is off by
ds = 2 (D + 8) eps max_v sum |h w| (products of halves 8 eps, additions 2 eps each); lse and
loss by 2 ds + 1e-5 + 8 eps |lse|; a value of a gradient by 4 ds + 1e-5 (p) + 1e-4 (additions)
of its terms' sum, and by 1e-5 in the norm.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 2.0**-24


def _check(h, w, y, weight, rows, items, backward=True):
    """`rows`, `items`: what is compared."""
    from paper_1410_8043_gb300 import esspt

    D = h.shape[1]
    head = esspt.SoftmaxHead(h.shape[0], w.shape[0], D, max_top=2)
    twice = torch.stack([torch.full_like(y, -1), y], 1).contiguous()
    results = [head.loss(h, w, y, weight=weight, backward=backward),
               head.distill(h, w, twice, torch.ones(twice.shape, device="cuda"), weight=weight, backward=backward)]
    head.poll()
    head.close()
    others = ~rows
    items = items & ~torch.zeros_like(items).index_fill_(0, y[others].long(), True)
    h64 = h[rows].double()
    full = w.double()
    s = h64 @ full[items].T
    drop = torch.logsumexp(h64 @ full.T, 1) - torch.logsumexp(s, 1)
    s_y = (h64 * full[y[rows].long()]).sum(1)
    lse = torch.logsumexp(h64 @ full.T, 1)
    prod = (h64.abs() @ full[items].abs().T).amax(1)
    assert int(rows.sum()) > 0 and int(items.sum()) > 0 and float(drop.abs().max()) < 10
    ds = 2 * (D + 8) * EPS * prod
    p = torch.exp(h64 @ full.T - lse[:, None])
    q = torch.zeros_like(p).scatter_(1, y[rows].long()[:, None], 1.0)
    wt = weight[rows].double()[:, None]
    want_h, mass_h = (wt * (p - q)) @ full, (wt.abs() * (p + q)) @ full.abs()
    want_w = (wt * (p - q)).T[items] @ h64
    mass_w = (wt.abs() * (p + q)).T[items] @ h64.abs()
    for r in results:
        tol = 2 * ds + 1e-5 + 8 * EPS * lse.abs()
        for got, want in ((r.lse[rows], lse), (r.loss[rows], lse - s_y)):
            err = (got.double() - want).abs()
            assert bool((err <= tol).all()), float((err / tol).max())
        if not backward:
            continue
        ep = 4 * ds + 1.1e-4
        for got, want, mass, e in ((r.grad_h[rows], want_h, mass_h, ep[:, None]), (r.grad_w[items], want_w, mass_w, ep.max())):
            err = (got.double() - want).abs()
            assert bool((err <= e * mass + 1e-37).all()), float((err / (e * mass + 1e-37)).max())
            assert float(err.norm()) <= 1e-5 * float(want.norm()), float(err.norm() / want.norm())


def _inputs(T, V, D, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    std = math.sqrt(2.0 / math.sqrt(D))
    h = torch.randn((T, D), generator=g, device="cuda") * std
    w = torch.randn((V, D), generator=g, device="cuda") * std
    y = torch.randint(0, V, (T,), generator=g, device="cuda").int()
    return h, w, y, torch.rand(T, generator=g, device="cuda") + 0.5


# Few rows; one tile; several; wide rows; a large problem.
SHAPES = [(6, 3000, 64), (200, 5000, 64), (300, 2000, 100), (260, 3001, 40), (200, 1500, 300), (150, 900, 512), (600, 150_001, 60)]


@pytest.mark.parametrize("factor", [1e4, 1e6, 1e8, 1e10, 1e13])
@pytest.mark.parametrize("T,V,D", SHAPES)
def test_one_row_of_h(T, V, D, factor):
    """A diverged row spoils nothing but what is its own."""
    h, w, y, weight = _inputs(T, V, D, 1)
    h[T // 2] *= factor
    rows = torch.arange(T, device="cuda") != T // 2
    items = torch.ones(V, dtype=torch.bool, device="cuda")
    items[torch.topk(h[T // 2].double() @ w.double().T, 1).indices] = False
    if factor < 1e6:  # (its p is not all at one item)
        s = h[T // 2].double() @ w.double().T
        items &= torch.exp(s - s.max()) < 1e-40
    _check(h, w, y, weight, rows, items)


@pytest.mark.parametrize("factor", [1e6, 1e8, 1e10, 1e13])
@pytest.mark.parametrize("T,V,D", SHAPES)
def test_one_item(T, V, D, factor):
    """A huge item draws some rows; the others do not see it."""
    h, w, y, weight = _inputs(T, V, D, 2)
    w[7] *= factor
    y = torch.where(y == 7, 8, y).int()
    score = h.double() @ w[7].double()
    rows = score < -1000
    weight[score.abs() <= 1000] = 0.0  # (neither drawn nor free of it)
    items = torch.ones(V, dtype=torch.bool, device="cuda")
    items[7] = False
    _check(h, w, y, weight, rows, items)


@pytest.mark.parametrize("backward", [True, False])
@pytest.mark.parametrize("mask", [-1e4, -1e6, -1e9, -1e15])
@pytest.mark.parametrize("T,V,D", SHAPES)
def test_items_masked_by_a_column(T, V, D, mask, backward):
    """A column that is one in H and very negative for items that are not to be scored."""
    h, w, y, weight = _inputs(T, V, D, 3)
    h[:, -1], w[:, -1] = 1.0, 0.1
    masked = torch.arange(V, device="cuda") % 17 == 3
    w[masked, -1] = mask
    y = torch.where(masked[y.long()], (y + 1) % V, y)
    y = torch.where(masked[y.long()], torch.zeros_like(y), y).int()
    _check(h, w, y, weight, torch.ones(T, dtype=torch.bool, device="cuda"), ~masked, backward)


@pytest.mark.parametrize("T,V,D", SHAPES)
def test_rows_and_items_of_every_size(T, V, D):
    """Sizes from 1e-8 to 1 among the rows and from 1e-6 to 1 among the items: small rows
    and items are as exact relative to themselves as large ones."""
    h, w, y, weight = _inputs(T, V, D, 4)
    g = torch.Generator("cuda").manual_seed(9)
    h *= 10.0 ** (-8 * torch.rand((T, 1), generator=g, device="cuda"))
    w *= 10.0 ** (-6 * torch.rand((V, 1), generator=g, device="cuda"))
    _check(h, w, y, weight, torch.ones(T, dtype=torch.bool, device="cuda"), torch.ones(V, dtype=torch.bool, device="cuda"))
