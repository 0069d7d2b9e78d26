"""Softmax gradients near a fit on the GPU, where they are small differences p - q and
what is left of a target comes from a long tail of tiny probabilities."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _head(*a, **kw):
    from paper_1410_8043_gb300 import esspt

    return esspt.SoftmaxHead(*a, **kw)


def _fitted(T, V, D, dtype, gap, seed):
    """Rows that score their own item `gap` above the others, whose scores have standard
    deviation 1.3; items share a mean, so that the tail's sum does not average out."""
    g = torch.Generator("cuda").manual_seed(seed)
    w = torch.randn((V, D), generator=g, device="cuda") * 0.3
    y = torch.randperm(V, generator=g, device="cuda")[:T]
    u = torch.nn.functional.normalize(torch.randn((T, D), generator=g, device="cuda"), dim=1)
    mean = torch.randn(D, generator=g, device="cuda") * 0.5
    w[y] = 5.0 * u
    w += mean
    h = u * (gap / 5.0)
    return h.to(TYPES[dtype]), w.to(TYPES[dtype]), y.int()


# What is allowed.  dh_t = sum_v p_tv w_v - w_y is taken relative to itself, not to its terms:
#   * a tail's p of about 2^-31 of the largest, kept 2^14 times as large in steps of 2^-24 at
#     most, is off by less than 2^-8 of itself, and by what is between scores: 1e-4;
#   * the target's p w and q w cancel.  Their sums are off by additions that truncate, 2^-23 of
#     the target's row each: 128 between two additions in fp32 (fp32 rows), 1024 (16-bit
#     rows), and 64 additions in fp32: 2.5e-5 and 1.3e-4 of |w_y| with the halves' 2^-22;
#   * 16-bit results are rounded, to their half-unit (of 2^-24 at least); bf16's tails too, and a
#     half-unit of theirs is within the 2^-8.
@pytest.mark.parametrize("kind", ["loss", "distill"])
@pytest.mark.parametrize("dtype,T,V,D", [("f32", 64, 1_000_003, 64), ("f16", 64, 1_000_003, 64), ("f32", 300, 400_001, 100),
                                         ("f32", 40, 500_009, 200), ("f16", 200, 500_009, 300),
                                         ("bf16", 64, 1_000_003, 64)])
def test_tail_of_a_large_catalogue(dtype, T, V, D, kind):
    gap = 21.5
    h, w, y = _fitted(T, V, D, dtype, gap, 5)
    head = _head(T, V, D, dtype=TYPES[dtype], max_top=2)
    if kind == "loss":
        r = head.loss(h, w, y)
    else:  # (the same target: an absent entry beside it)
        ids = torch.stack([torch.full_like(y, -1), y], 1).contiguous()
        r = head.distill(h, w, ids, torch.zeros(ids.shape, device="cuda"))
    head.poll()
    w64 = w.double()
    for rows in torch.arange(T, device="cuda").split(50):
        s = h[rows].double() @ w64.T
        lse = torch.logsumexp(s, 1)
        p = torch.exp(s - lse[:, None])
        p[torch.arange(len(rows)), y[rows].long()] = 0.0
        rest = p.sum(1, keepdim=True)
        want = p @ w64 - rest * w64[y[rows].long()]
        assert 1e-5 < float(rest.min()) and float(rest.max()) < 1e-2
        err = (r.grad_h[rows].double() - want).norm(dim=1)
        bound = (2.0**-8 + 1e-4) * want.norm(dim=1) + (2.5e-5 if dtype == "f32" else 1.3e-4) * w64[y[rows].long()].norm(dim=1)
        if dtype != "f32":
            bound = bound + torch.finfo(TYPES[dtype]).eps / 2 * want.norm(dim=1) + 2.0**-25 * math.sqrt(D)
        assert bool((err <= bound).all()), float((err / bound).max())


EPS = 2.0**-24


def _dw(h, w, ids, weight, items):
    """Rows `items` of dw in fp64, their terms' absolute sums, and the largest sum of a score's."""
    h64, w64, at = h.double(), w.double(), ids.long()
    s = h64 @ w64.T
    p = torch.exp(s - torch.logsumexp(s, 1, keepdim=True))[:, items]
    q = (at[:, None] == items[None]).double()
    g = weight.double()[:, None] * (p - q)
    mass = (weight.double().abs()[:, None] * (p + q)).T @ h64.abs()
    return g.T @ h64, mass, float((h64.abs() @ w64.abs().T).max())


def _check_items(r, h, w, ids, weight, items, dtype, D):
    """Every value relative to its own terms: p is off by what its score is (2 ds: 8 eps a
    product, 2 eps an addition), by exponentials and by halves of 11 bits (1e-5; 16-bit
    rows: the type's half-unit), sums by 1e-4, the result by its rounding."""
    want, mass, prod = _dw(h, w, ids, weight, items)
    half = 2.0**-24 if dtype == "f32" else torch.finfo(TYPES[dtype]).eps / 2
    ep = 4 * (D + 8) * EPS * prod + 1e-5 + half + 1e-4
    err = (r.grad_w[items].double() - want).abs()
    bound = ep * mass + half * want.abs() + (0 if dtype == "f32" else 2.0**-25)
    assert bool((err <= bound).all()), float((err / bound).max())


@pytest.mark.parametrize("T,V,D,gap", [(64, 1_000_003, 64, 28.0), (300, 100_003, 150, 40.0)])
def test_items_that_are_nobodys_target(T, V, D, gap):
    """Their gradients are sums of probabilities of 2^-40 and less: as good, relative to
    themselves, as any other's."""
    h, w, y = _fitted(T, V, D, "f32", gap, 6)
    head = _head(T, V, D)
    weight = torch.ones(T, device="cuda")
    r = head.loss(h, w, y, weight=weight)
    head.poll()
    items = torch.arange(0, V, max(1, V // 2000), device="cuda")
    items = items[~torch.isin(items, y.long())]
    _check_items(r, h, w, y, weight, items, "f32", D)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D", [(200, 3000, 64), (700, 9000, 150), (6, 3000, 64)])
def test_one_weight_far_above_the_others(T, V, D, dtype, sign):
    """A row with a weight of 1e8 that is fitted (p of its target near one): items that have
    nothing of it keep the gradients of the other rows."""
    g = torch.Generator("cuda").manual_seed(T)
    w = torch.randn((V, D), generator=g, device="cuda") * 0.5
    u = torch.nn.functional.normalize(torch.randn(D, generator=g, device="cuda"), dim=0)
    h = torch.randn((T, D), generator=g, device="cuda") * 0.3
    y = torch.randint(1, V, (T,), generator=g, device="cuda").int()
    w[0], h[3], y[3] = 8.0 * u, 11.0 * u, 0  # 88 above the others' mean, their deviation is 5.5
    h, w = h.to(TYPES[dtype]), w.to(TYPES[dtype])
    weight = torch.rand(T, generator=g, device="cuda") + 0.5
    weight[3] = 1e8 * sign
    weight[4] *= -1
    head = _head(T, V, D, dtype=TYPES[dtype])
    r = head.loss(h, w, y, weight=weight)
    head.poll()
    _check_items(r, h, w, y, weight, torch.arange(1, V, device="cuda"), dtype, D)
