"""Embedding lookup and its gradient on the GPU, against the definition in fp64.

Tolerances, eps = 2^-24: a looked-up value is a product rounded to fp32 and then to its type, so off by
eps and the type's half unit; a gradient of m terms takes m additions of any order and one product, each off by eps of
the sum of magnitudes, and the result's rounding.  Subnormal results are off by half their spacing.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

EPS = 2.0**-24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {name: torch.finfo(t).eps / 2 for name, t in TYPES.items()}
TINY = {"f32": 2.0**-149, "bf16": 2.0**-133, "f16": 2.0**-24}


def _esspt():
    from paper_1410_8043_gb300 import esspt

    return esspt


def _inputs(T, V, D, dtype, seed, pad=0.2, hot=0.5):
    """Ids with one popular row, padding with NaN gradients; rows of a wider buffer for odd seeds."""
    g = torch.Generator("cuda").manual_seed(seed)
    wide = D + (seed % 2) * 3
    w = torch.randn((V, wide), generator=g, device="cuda").to(TYPES[dtype])[:, :D]
    grad = torch.randn((T, wide), generator=g, device="cuda").to(TYPES[dtype])[:, :D]
    ids = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    ids[torch.rand(T, generator=g, device="cuda") < hot] = V // 2
    drop = torch.rand(T, generator=g, device="cuda") < pad
    ids[drop] = -1 - torch.randint(0, 5, (T,), generator=g, device="cuda", dtype=torch.int32)[drop]
    grad[drop] = math.nan
    return w, ids, grad


def _check_lookup(out, w, ids, scale, dtype):
    want = torch.where((ids >= 0)[:, None], w.double()[ids.long().clamp(min=0)] * scale, 0.0)
    tol = (HALF[dtype] * (1 + EPS) + EPS) * want.abs() + TINY[dtype]
    assert bool(((out.double() - want).abs() <= tol).all())
    assert bool((out[ids < 0] == 0).all())


def _check_gradient(out, ids, grad, scale, dtype, V, before=None):
    kept = ids >= 0
    at, rows = ids[kept].long(), grad[kept].double()
    zero = torch.zeros((V, grad.shape[1]), dtype=torch.float64, device="cuda")
    count = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, at, torch.ones_like(at, dtype=torch.float64))[:, None]
    want = zero.index_add(0, at, rows) * scale
    mass = zero.index_add(0, at, rows.abs()) * abs(scale)
    if before is not None:
        want, mass = want + before.double(), mass + before.double().abs()
    tol = (count + 2) * EPS * mass + HALF[dtype] * (1 + 1e-3) * want.abs() + TINY[dtype]
    err = (out.double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    untouched = (count == 0)[:, 0]
    assert bool((out[untouched] == (0 if before is None else before[untouched])).all())


# One token to many, one row to many; widths at and around vectors, a warp's 32 of them, and the widest.
SHAPES = [(1, 1, 1), (1, 1000, 64), (2, 3, 5), (31, 7, 8), (33, 1, 100), (97, 1000, 16), (127, 50, 129), (1000, 40, 257),
          (513, 300, 33), (2049, 5000, 12), (4097, 30_000, 64), (300, 100, 8192), (77, 12, 8191), (20_001, 700, 100),
          (16_384, 50_021, 24), (16_385, 3, 40), (70_001, 5000, 48), (40_000, 200_000, 17), (66_000, 66_000, 64), (300_000, 1000, 9)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T, V, D", SHAPES)
def test_against_fp64(T, V, D, dtype):
    seed = T + V + D
    w, ids, grad = _inputs(T, V, D, dtype, seed)
    scale = 1.0 if seed % 3 else math.sqrt(D)
    em = _esspt().Embedding(T, V, D, dtype=TYPES[dtype])
    _check_lookup(em.lookup(w, ids, scale=scale), w, ids, scale, dtype)
    first = em.gradient(ids, grad, scale=scale)
    _check_gradient(first, ids, grad, scale, dtype, V)
    again = em.gradient(ids, grad, scale=scale, grad_w=torch.full_like(first, math.nan))
    assert torch.equal(first, again)  # the same bits, and every row is written
    before = torch.randn((V, D), device="cuda").to(TYPES[dtype])
    got = em.gradient(ids, grad, scale=scale, grad_w=before.clone(), accumulate=True)
    _check_gradient(got, ids, grad, scale, dtype, V, before)
    em.poll()
    em.close()


@pytest.mark.parametrize("ids", ["same", "padding", "distinct", "sorted", "last"])
@pytest.mark.parametrize("T, V, D", [(1000, 1000, 20), (30_000, 30_000, 64), (50_000, 60_000, 8)])
def test_orders_of_ids(T, V, D, ids):
    """All one row, all padding, every row once, in order, the table's last row."""
    g = torch.Generator("cuda").manual_seed(1)
    at = {"same": torch.full((T,), 3), "padding": torch.full((T,), -1), "distinct": torch.randperm(V)[:T],
          "sorted": torch.arange(T) // 7, "last": torch.full((T,), V - 1)}[ids].to(torch.int32).cuda()
    grad = torch.randn((T, D), generator=g, device="cuda")
    em = _esspt().Embedding(T, V, D)
    _check_gradient(em.gradient(at, grad, scale=-0.5), at, grad, -0.5, "f32", V)
    before = torch.randn((V, D), generator=g, device="cuda")
    _check_gradient(em.gradient(at, grad, grad_w=before.clone(), accumulate=True), at, grad, 1.0, "f32", V, before)
    em.close()


@pytest.mark.parametrize("T", [40, 50_000])
def test_no_tokens_and_fewer_than_the_most(T):
    em = _esspt().Embedding(T, 50, 6)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    rows = torch.empty((0, 6), device="cuda")
    w = torch.randn((50, 6), device="cuda")
    assert em.lookup(w, none).shape == (0, 6)
    assert bool((em.gradient(none, rows, grad_w=torch.full_like(w, 7.0)) == 0).all())
    assert torch.equal(em.gradient(none, rows, grad_w=w.clone(), accumulate=True), w)
    _, ids, grad = _inputs(17, 50, 6, "f32", 4)
    _check_gradient(em.gradient(ids, grad), ids, grad, 1.0, "f32", 50)
    em.close()


@pytest.mark.parametrize("T", [90, 40_000])
def test_ids_outside_the_table(T):
    """Padding for the results, an error for poll, which clears it; 64-bit ids stay outside."""
    e = _esspt()
    em = e.Embedding(T, 50, 8)
    w, ids, grad = _inputs(T, 50, 8, "f32", 6)
    bad = ids.clone()
    bad[3] = 50
    held = ids.clone()
    held[3] = -1
    for call in (lambda i: em.lookup(w, i), lambda i: em.gradient(i, grad)):
        got = call(bad)
        with pytest.raises(e.EssptError) as err:
            em.poll()
        assert err.value.status == e.EINVAL
        em.poll()
        assert torch.equal(got, call(held))
    far = ids.long()
    far[3] = 2**32 + 1
    assert torch.equal(em.lookup(w, far), em.lookup(w, held))
    em.close()


def test_sorts_of_every_length_fit_the_workspace():
    """Fewer tokens may take more tiles of the sort than the most do: 2.49M of 10M."""
    T, V, D = 10_000_000, 3000, 1
    em = _esspt().Embedding(T, V, D)
    guard = torch.full((1 << 20,), 7, dtype=torch.uint8, device="cuda")
    for n in (2_490_368, 2_490_369, T, 20_000):
        ids = torch.randint(-1, V, (n,), dtype=torch.int32, device="cuda")
        got = em.gradient(ids, torch.ones((n, 1), device="cuda"))
        assert torch.equal(got[:, 0].long(), torch.bincount(ids.long() + 1, minlength=V + 1)[1:])
    assert bool((guard == 7).all())
    em.poll()
    em.close()


def test_special_values():
    """Infinity and NaN go to their own row alone; fp16 sums past its range are infinite."""
    em = _esspt().Embedding(6, 9, 8, dtype=torch.float16)
    ids = torch.tensor([2, 5, 2, 7, 0, 8], dtype=torch.int32, device="cuda")
    grad = torch.ones((6, 8), dtype=torch.float16, device="cuda")
    grad[0], grad[2], grad[3, 1], grad[4, 0] = 60_000.0, 60_000.0, math.nan, -math.inf
    out = em.gradient(ids, grad)
    assert bool((out[2] == math.inf).all()) and bool(torch.isnan(out[7, 1])) and float(out[0, 0]) == -math.inf
    out[2], out[7, 1], out[0, 0] = 0, 0, 0
    assert bool(torch.isfinite(out).all())
    half = em.gradient(ids, grad, scale=0.25)
    assert bool((half[2] == 30_000.0).all())  # (the sum itself is fp32)
    em.close()


def test_offsets_past_32_bits():
    """A table of 2^31 values and more: its last rows."""
    V, D, T = 33_600_000, 64, 40_000
    w = torch.zeros((V, D), dtype=torch.bfloat16, device="cuda")
    w[-5:] = torch.randn((5, D), device="cuda").to(torch.bfloat16)
    em = _esspt().Embedding(T, V, D, dtype=torch.bfloat16)
    ids = torch.randint(V - 5, V, (T,), dtype=torch.int32, device="cuda")
    assert torch.equal(em.lookup(w, ids), w[ids.long()])
    grad = torch.ones((T, D), dtype=torch.bfloat16, device="cuda")
    for n in (300, T):
        got = em.gradient(ids[:n], grad[:n], scale=1 / 1024)
        count = torch.bincount(ids[:n].long() - (V - 5), minlength=5)
        assert torch.equal(got[-5:], (count / 1024).to(torch.bfloat16)[:, None].expand(5, D))
        assert int(torch.count_nonzero(got[:-5])) == 0
    em.close()


@pytest.mark.parametrize("T", [200, 30_000])
def test_another_stream_and_a_graph(T):
    """Calls from a stream that is not the handle's, and a captured call on inputs that change."""
    side = torch.cuda.Stream()
    w, ids, grad = _inputs(T, 500, 24, "f32", 2)
    em = _esspt().Embedding(T, 500, 24, stream=side)
    ids2 = ids.flip(0).contiguous()
    grad2 = grad.flip(0).contiguous()
    _check_lookup(em.lookup(w, ids), w, ids, 1.0, "f32")
    _check_gradient(em.gradient(ids, grad), ids, grad, 1.0, "f32", 500)
    a, b, total = ids.clone(), grad.clone(), torch.zeros((500, 24), device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        rows = em.lookup(w, a)
        out = em.gradient(a, b)
        em.gradient(a, b, grad_w=total, accumulate=True)
    for x, y in ((ids, grad), (ids2, grad2), (ids, grad)):
        a.copy_(x), b.copy_(y), total.fill_(1.0)
        graph.replay()
        _check_lookup(rows, w, x, 1.0, "f32")
        _check_gradient(out, x, y, 1.0, "f32", 500)
        _check_gradient(total, x, y, 1.0, "f32", 500, torch.ones_like(total))
    em.poll()
    em.close()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T, V, D", [(40, 30, 33), (40, 30, 64), (3001, 500, 7), (30_000, 700, 101), (30_000, 700, 16)])
@pytest.mark.parametrize("shift", [1, 2, 4])
def test_addresses_off_the_vectors(T, V, D, shift, dtype):
    """Tables, gradients and results that begin anywhere in memory, and nothing written beside them."""
    w, ids, grad = _inputs(T, V, D, dtype, 2 * (T + D))
    em = _esspt().Embedding(T, V, D, dtype=TYPES[dtype])

    def placed(x, rows, cols):
        buf = torch.full((rows * cols + 16,), 7.0, dtype=TYPES[dtype], device="cuda")
        view = buf[shift:shift + rows * cols].view(rows, cols)
        if x is not None:
            view.copy_(x)
        return buf, view

    _, w2 = placed(w, V, D)
    _, grad2 = placed(grad, T, D)
    rows, out = placed(None, T, D)
    _check_lookup(em.lookup(w2, ids, scale=3.0, out=out), w, ids, 3.0, dtype)
    table, total = placed(None, V, D)
    _check_gradient(em.gradient(ids, grad2, grad_w=total), ids, grad, 1.0, dtype, V)
    for buf, n in ((rows, T * D), (table, V * D)):
        assert bool((buf[:shift] == 7).all()) and bool((buf[shift + n:] == 7).all())
    em.close()


def test_zeros_beside_the_sort_in_a_graph():
    """A gradient large enough for the handle's second stream, captured, onto a table of NaN."""
    T, V, D = 20_000, 300_000, 64
    side = torch.cuda.Stream()
    em = _esspt().Embedding(T, V, D, stream=side)
    _, ids, grad = _inputs(T, V, D, "f32", 8)
    out = torch.full((V, D), math.nan, device="cuda")
    a, b = ids.clone(), grad.clone()
    _check_gradient(em.gradient(ids, grad, grad_w=out), ids, grad, 1.0, "f32", V)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        em.gradient(a, b, grad_w=out)
    for x, y in ((ids, grad), (ids.flip(0), grad.flip(0)), (ids, grad)):
        a.copy_(x), b.copy_(y), out.fill_(math.nan)
        graph.replay()
        _check_gradient(out, x, y, 1.0, "f32", V)
    torch.cuda.synchronize()
    em.close()


def test_refusals():
    e = _esspt()
    em = e.Embedding(8, 10, 4, backward=False)
    w, ids = torch.zeros((10, 4), device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    grad = torch.zeros((8, 4), device="cuda")
    for call in (
        lambda: e.Embedding(0, 10, 4), lambda: e.Embedding(8, 10, 4, dtype=torch.float64),
        lambda: em.gradient(ids, grad), lambda: em.lookup(w[:9], ids), lambda: em.lookup(w.half(), ids),
        lambda: em.lookup(w.cpu(), ids), lambda: em.lookup(w, ids.cpu()), lambda: em.lookup(w, ids.float()),
        lambda: em.lookup(w, ids[None]), lambda: em.lookup(w, torch.zeros(9, dtype=torch.int32, device="cuda")),
        lambda: em.lookup(w, ids, scale=math.inf), lambda: em.lookup(w, ids, out=torch.zeros((8, 5), device="cuda")),
        lambda: em.lookup(w, ids, out=torch.zeros((4, 8), device="cuda").T),
    ):
        with pytest.raises(e.EssptError):
            call()
    em.close()
    em = e.Embedding(8, 10, 4)
    for call in (lambda: em.gradient(ids, grad[:7]), lambda: em.gradient(ids, grad, accumulate=True),
                 lambda: em.gradient(ids, grad, scale=math.nan), lambda: em.gradient(ids, grad, grad_w=w[:9])):
        with pytest.raises(e.EssptError):
            call()
    assert torch.equal(em.lookup(w.T.contiguous().T + 1, ids), grad + 1)  # another layout is copied
    em.close()


# -- sums that no order rounds ----------------------------------------------------


def _whole(T, V, D, dtype, at, seed, stride=0):
    """Gradients and a table of whole numbers up to 8, NaN at padding; what is to come out of them in fp64, half of the sums."""
    g = torch.Generator("cuda").manual_seed(seed)
    grad = torch.randint(-8, 9, (T, D + stride), generator=g, device="cuda").to(TYPES[dtype])[:, :D]
    grad[at < 0] = math.nan
    before = torch.randint(-8, 9, (V, D), generator=g, device="cuda").to(TYPES[dtype])
    kept = at >= 0
    sums = torch.zeros((V, D), dtype=torch.float64, device="cuda").index_add_(0, at[kept].long(), grad[kept].double())
    return grad, before, 0.5 * sums


def _check_whole(em, at, grad, before, want, dtype):
    """Sums stay below 2^24 and are whole: fp32 holds them in any order, and the result is rounded once, to its type."""
    assert float(want.abs().max()) < 2**22
    t = TYPES[dtype]
    assert torch.equal(em.gradient(at, grad, scale=0.5, grad_w=torch.full_like(before, math.nan)), want.float().to(t))
    got = em.gradient(at, grad, scale=0.5, grad_w=before.clone(), accumulate=True)
    assert torch.equal(got, (before.double() + want).float().to(t))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T, V, D", SHAPES + [(120_000, 1000, 9), (200_003, 40, 100), (250_000, 3, 64), (500_000, 300_000, 40)])
def test_no_token_is_lost(T, V, D, dtype):
    """Every shape with one popular row (up to half of the tokens), equal to the last bit: what bounds the kernels'
    rounding grows with a row's tokens and would hide one that is left out or added twice."""
    _, at, _ = _inputs(T, V, 1, dtype, T + V + D)
    grad, before, want = _whole(T, V, D, dtype, at, T, stride=(0, 3, 8)[(T + D) % 3])
    em = _esspt().Embedding(T, V, D, dtype=TYPES[dtype])
    _check_whole(em, at, grad, before, want, dtype)
    em.poll()
    em.close()


@pytest.mark.parametrize("ids", ["same", "two", "padding", "distinct", "sorted", "blocks", "last"])
@pytest.mark.parametrize("T, V, D", [(3000, 4000, 20), (16_384, 16_384, 7), (30_000, 30_000, 64), (50_000, 60_000, 8), (130_000, 130_000, 33)])
def test_no_token_is_lost_in_any_order(T, V, D, ids):
    """Rows of all tokens (as many parts as there are blocks), runs that end at and beside the blocks' ends."""
    g = torch.Generator().manual_seed(T)
    at = {"same": torch.full((T,), 3), "two": torch.arange(T) % 2 * (V - 1), "padding": torch.full((T,), -1), "distinct": torch.randperm(V, generator=g)[:T],
          "sorted": torch.arange(T) // 7, "blocks": (torch.arange(T) + 1) // 256 // 2,
          "last": torch.where(torch.rand(T, generator=g) < 0.3, -1, V - 1)}[ids].to(torch.int32).cuda()
    grad, before, want = _whole(T, V, D, "f32", at, T + 1)
    em = _esspt().Embedding(T, V, D)
    _check_whole(em, at, grad, before, want, "f32")
    em.close()


@pytest.mark.parametrize("T, V, D", [(40_000, 700, 64), (300_000, 2**20, 4), (1_000_003, 5000, 1), (2_500_000, 3000, 2), (17_000, 2**22 + 1, 16), (16_400, 9, 8192)])
def test_nothing_behind_the_workspace_is_written(T, V, D):
    """The library's handle on a part of a buffer, the bytes right behind the workspace kept in view, for as many tokens as
    the handle takes and fewer."""
    import ctypes

    e = _esspt()
    L = e.lib()
    cfg = e.EmbedConfig(T, V, D, 0, 1, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    size = L.esspt_embed_workspace_bytes(ctypes.byref(cfg))
    tail = 8 << 20
    buf = torch.full((size + tail + 256,), 7, dtype=torch.uint8, device="cuda")
    skip = -buf.data_ptr() % 256
    h = ctypes.c_void_p()
    assert L.esspt_embed_create(ctypes.byref(cfg), buf.data_ptr() + skip, size, ctypes.byref(h)) == e.OK
    total = torch.empty((V, D), device="cuda")
    for n in sorted({T, T - 1, T // 2, T * 3 // 4, T // 3 + 1, 16_385, 2049}):
        at = torch.randint(-1, V, (n,), dtype=torch.int32, device="cuda")
        grad = torch.ones((n, D), device="cuda")
        for accumulate in (0, 1):
            st = L.esspt_embed_gradient(h, at.data_ptr(), grad.data_ptr(), D, n, 1.0, accumulate, total.data_ptr())
            assert st == e.OK, L.esspt_embed_last_error(h)
        count = torch.bincount(at.long() + 1, minlength=V + 1)[1:]
        assert torch.equal(total, (2 * count).float()[:, None].expand(V, D))
        assert bool((buf[:skip] == 7).all()) and bool((buf[skip + size:] == 7).all())
    assert L.esspt_embed_poll(h) == e.OK and L.esspt_embed_destroy(h) == e.OK
