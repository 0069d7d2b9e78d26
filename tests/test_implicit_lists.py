"""A teacher's lists by pieces of the catalogue are those of the whole (CPU)."""
import pytest
import torch


@pytest.mark.parametrize("M,top,piece", [(1000, 20, 65536), (1000, 20, 128), (1000, 20, 7), (30, 50, 8), (1, 3, 1), (257, 257, 256)])
def test_top_scores(M, top, piece):
    from paper_1410_8043_gb300.implicit import top_scores

    g = torch.Generator().manual_seed(M)
    h, r = torch.randn((9, 6), generator=g, dtype=torch.float64), torch.randn((M, 6), generator=g, dtype=torch.float64)
    items, values = top_scores(h, r, top, piece)
    want = torch.topk(h @ r.T, min(top, M), dim=1)
    assert items.dtype is torch.int32 and items.shape == want.indices.shape
    assert torch.allclose(values, want.values, rtol=0, atol=1e-12)
    assert torch.equal(items.long(), want.indices)
