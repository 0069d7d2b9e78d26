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
