"""Teacher's lists that name an item more than once, p about 0.99 (GPU): q is the sum of its
shares, and p of the item comes off once."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# As for one entry near a fit: twice the half-unit of the type (p of the others, the result).  Of
# 16-bit rows that is asked of nine rows of a gradient in ten, for a target's p may round the
# other way in the product than where it is taken off: the scores there differ by about
# sqrt(D) eps sum |h w|, 10^-5, a fiftieth of fp16's unit.  Additions of 16 products each truncate,
# 2^-23 of the terms at most, 1024 times before fp32 takes over.
BOUND = {"f32": 1e-5, "bf16": 2.0**-7, "f16": 2.0**-10}


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("top,places", [(2, (0, 1)), (9, (0, 1, 2, 3, 4, 5, 7, 8)), (40, (3, 39)), (100, (0, 31, 32, 64, 99)),
                                        (300, tuple(range(0, 300, 7)))])
@pytest.mark.parametrize("T,V", [(8, 2000), (60, 2000), (300, 2000), (900, 66_000)])
def test_item_named_again(T, V, top, places, dtype):
    D = 64
    g = torch.Generator("cuda").manual_seed(top)
    w = (torch.randn((V, D), generator=g, device="cuda") * 0.5).to(TYPES[dtype])
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    h = (w[y].float() * 0.9).to(w.dtype)
    ids = torch.randint(0, V, (T, top), generator=g, device="cuda").int()
    z = torch.full((T, top), -30.0, device="cuda")  # (a share of 1e-13)
    ids[:, list(places)] = y[:, None].int()
    z[:, list(places)] = 2.0 * torch.rand((T, len(places)), generator=g, device="cuda")
    ids[:, [k for k in range(top) if k not in places][::2]] = -1
    weight = torch.rand(T, generator=g, device="cuda") + 0.5

    from paper_1410_8043_gb300 import esspt

    head = esspt.SoftmaxHead(T, V, D, dtype=w.dtype, max_top=top)
    r = head.distill(h, w, ids, z, weight=weight)
    head.poll()
    h64, w64 = h.double(), w.double()
    p = torch.softmax(h64 @ w64.T, 1)
    q = torch.softmax(torch.where(ids >= 0, z.double(), -float("inf")), 1)
    q = torch.zeros_like(p).scatter_add_(1, ids.long().clamp(min=0), torch.where(ids >= 0, q, 0.0))
    g, terms = (p - q) * weight.double()[:, None], (p + q) * weight.double()[:, None]
    for got, want, size in ((r.grad_h, g @ w64, terms @ w64.abs()), (r.grad_w, g.T @ h64, terms.T @ h64.abs())):
        if dtype == "f32":  # each share is rounded, and so is every difference: eps of the terms
            bound = BOUND[dtype] * float(want.norm()) + (len(places) + 8) * 2.0**-24 * float(size.norm())
            assert float((got.double() - want).norm()) <= bound
            continue
        adds = min(1024, (V if want.shape[0] == T else T) // 16 + 1)
        if want.shape[0] == V:  # items that are targets
            got, want, size = (x[y.unique()] for x in (got, want, size))
        err = (got.double() - want).norm(dim=1)
        bound = BOUND[dtype] * want.norm(dim=1) + adds * 2.0**-23 * size.norm(dim=1) + 2.0**-25 * D**0.5
        assert float((err <= bound).double().mean()) >= 0.9, float((err / bound).quantile(0.9))
