"""Scores of many thousand millions on the GPU, where fp32 has no fraction left: a row's
probability is all at its best item, and nothing becomes NaN."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 2.0**-24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.mark.parametrize("best", ["target", "another"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("size", [3e4, 1e7, 1e9, 1e12])
@pytest.mark.parametrize("T,V,D", [(8, 700, 64), (200, 700, 64), (300, 2000, 100), (150, 900, 300), (140, 500, 512), (512, 150_001, 40)])
def test_best_item_takes_all(T, V, D, size, dtype, best):
    """Every other row has scores of `size`, its best item far above the next; the others
    are ordinary.  Losses hold to fp32 rounding of the scores (ds = 2 (D + 8) eps max sum
    |h w|); gradients to the type's rounding of each term: a large row's are its best item's
    and its target's alone."""
    g = torch.Generator("cuda").manual_seed(T + D)
    h = torch.randn((T, D), generator=g, device="cuda")
    w = torch.randn((V, D), generator=g, device="cuda")
    u = torch.nn.functional.normalize(torch.randn(D, generator=g, device="cuda"), dim=0)
    w[0] = 3.0 * u + w[0] * 0.1
    w[1:] -= 0.5 * torch.outer(w[1:] @ u, u)
    if dtype == "f16":  # (65504 at most: both sides large)
        a, c = min(math.sqrt(size), 2e3), min(size / math.sqrt(size), 2e3)
    else:
        a, c = size, 1.0
    large = torch.arange(T, device="cuda") % 2 == 1
    h = torch.where(large[:, None], (h * 0.02 + 4.0 * u) * a, h * (0.3 / c)).to(TYPES[dtype])
    w = (w * c).to(TYPES[dtype])
    y = torch.randint(1, V, (T,), generator=g, device="cuda").int()
    if best == "target":
        y[large] = 0
    weight = torch.rand(T, generator=g, device="cuda") + 0.5

    from paper_1410_8043_gb300 import esspt

    head = esspt.SoftmaxHead(T, V, D, dtype=TYPES[dtype], max_top=2)
    ids = torch.stack([y, torch.full_like(y, -1)], 1).contiguous()
    results = [head.loss(h, w, y, weight=weight), head.distill(h, w, ids, torch.zeros(ids.shape, device="cuda"), weight=weight)]
    head.poll()
    h64, w64 = h.double(), w.double()
    s = h64 @ w64.T
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None])
    assert float((p[large][:, 0] - 1).abs().max()) < 1e-30
    q = torch.zeros_like(p).scatter_(1, y.long()[:, None], 1.0)
    loss = lse - s.gather(1, y.long()[:, None])[:, 0]
    ds = 2 * (D + 8) * EPS * (h64.abs() @ w64.abs().T).amax(1)
    wt = weight.double()[:, None]
    half = EPS if dtype == "f32" else torch.finfo(TYPES[dtype]).eps / 2
    ep = torch.where(large, 1e-4, 4 * ds + 1.1e-4)[:, None] + half
    top = 65504.0 if dtype == "f16" else math.inf
    for r in results:
        for got, want in ((r.lse, lse), (r.loss, loss)):
            tol = 2 * ds + 1e-5 + 8 * EPS * lse.abs()
            assert bool(((got.double() - want).abs() <= tol).all())
        for got, want, mass in ((r.grad_h, (wt * (p - q)) @ w64, (ep * wt * (p + q)) @ w64.abs()),
                                (r.grad_w, (wt * (p - q)).T @ h64, (ep * wt * (p + q)).T @ h64.abs())):
            fits = want.abs() < top / 2
            err = (got.double() - want).abs()
            bound = mass + half * want.abs() + 2.0**-24
            assert bool(torch.isfinite(got)[fits].all())
            assert bool((err <= bound)[fits].all()), float((err / bound)[fits].max())
