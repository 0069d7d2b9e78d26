"""The softmax operators' ways of large problems and of batches of 9 to 128 rows over a large
catalogue (GPU), with the tolerances of the operators' other tests."""
import math

import pytest
import torch
from test_gpu_softmax import TYPES, _check, _esspt, _inputs, _reference, _run

pytestmark = pytest.mark.gpu


# More than 2^24 scores: by tiles, whatever the rows' number.
@pytest.mark.parametrize("kind,top", [("loss", 1), ("distill", 5), ("distill", 70)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D", [(17, 1_000_001, 24), (64, 300_001, 100), (100, 200_003, 64), (128, 140_001, 61),
                                   (120, 150_001, 300)])
def test_some_rows_over_a_large_catalogue(T, V, D, dtype, kind, top):
    h, w, ids, z, weight = _inputs(T, V, D, dtype, top, T + V + D + top)
    zz = torch.zeros_like(z) if kind == "loss" else z
    ref = _reference(h, w, ids, zz, weight, 1.0)
    _check(_run(kind, h, w, ids, z, weight, 1.0), ref, dtype, D, 1.0)
    _check(_run(kind, h, w, ids, z, weight, 1.0, backward=False), ref, dtype, D, 1.0)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D", [(600, 150_001, 40), (1700, 40_003, 130), (200, 900, 40)])
def test_one_row_that_is_no_number(T, V, D, dtype, bad):
    """Its loss, dh and (with the formula) dw are NaN; the other rows are what they are
    without it, and so are they when its value stands in the weight."""
    h, w, ids, z, weight = _inputs(T, V, D, dtype, 3, 7, pad=0.0)
    row = T // 3
    without = ids.clone()
    without[row] = -1
    ref = _reference(h, w, without, z, weight, 1.0)
    for where in ("h", "weight"):
        h2, weight2 = h.clone(), weight.clone()
        if where == "h":
            h2[row, 3] = bad
        else:
            weight2[row] = bad
        r = _run("distill", h2, w, ids, z, weight2, 1.0)
        assert bool(r.loss[row].isnan()) == (where == "h")
        assert not bool(r.grad_h[row].isfinite().all()) and not bool(r.grad_w.isfinite().all())
        mine = torch.arange(T, device="cuda") == row
        rest = _esspt().SoftmaxResult(r.loss.masked_fill(mine, 0.0), r.lse.masked_fill(mine, 0.0),
                                      r.grad_h.masked_fill(mine[:, None], 0.0), ref["grad_w"].to(TYPES[dtype]))
        _check(rest, ref, dtype, D, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_an_item_that_is_no_number(dtype):
    T, V, D = 600, 150_001, 40
    h, w, ids, z, weight = _inputs(T, V, D, dtype, 1, 8, pad=0.0)
    w[V - 1, D - 1] = math.nan
    for backward in (True, False):
        r = _run("loss", h, w, ids, z, weight, 1.0, backward=backward)
        assert bool(r.loss.isnan().all()) and bool(r.lse.isnan().all())
    assert bool(r.grad_h is None)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D,top", [(2000, 60_001, 64, 5), (300, 200_003, 100, 1), (8195, 9001, 40, 300)])
def test_same_bits_twice_in_large_problems(T, V, D, top, dtype):
    h, w, ids, z, weight = _inputs(T, V, D, dtype, top, 43)
    a, b = (_run("distill", h, w, ids, z, weight, 1.0) for _ in range(2))
    assert all(torch.equal(x, y) for x, y in zip(a, b))
