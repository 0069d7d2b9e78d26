"""Layer norm on the GPU, forward and backward, against the definition in fp64.

Tolerances, eps = 2^-24.  A sum over a row goes through at most 64 additions in a thread, 5 in a warp and 32 across
warps: 101, taken as 128 eps of the sum of magnitudes.  So
  mean: 128 eps mean|x|;  x - mean: that and eps of itself;  rstd: half of the variance's 2 eps + 128 eps, a square
  root, a quotient: 70 eps, and half the square of the mean's error in standard deviations;
  y: |w| (the error of x - mean) rstd + 72 eps |x^ w| + 2 eps (|x^ w| + |b|) + the rounding of the result;
  dx, from the statistics that the call is given: x^ is off by 3 eps, sums by 128 + 8 eps of their terms' magnitudes:
  140 eps rstd (|g| + mean|g| + |x^| mean|g x^|) + the rounding;
  dw, db: a thread's rows (600 at most here), up to 256 groups of a block, 128 blocks of a warp, 8 warps: fewer
  than n of them are not empty: min(n, 992) + 8 eps of the sum of magnitudes + the rounding.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

EPS = 2.0**-24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {name: torch.finfo(t).eps / 2 for name, t in TYPES.items()}
TINY = {"f32": 2.0**-140, "bf16": 2.0**-133, "f16": 2.0**-24}


def _esspt():
    from paper_1410_8043_gb300 import esspt

    return esspt


def _inputs(n, D, dtype, wtype, seed, stride=0, offset=1.0):
    g = torch.Generator("cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x = (r(n, D + stride) + offset * r(n, 1)).to(TYPES[dtype])[:, :D]
    dy = r(n, D + stride).to(TYPES[dtype])[:, :D]
    return x, dy, (1 + 0.3 * r(D)).to(TYPES[wtype]), (0.3 * r(D)).to(TYPES[wtype])


def _check_forward(r, x, w, b, dtype, eps=1e-5):
    x, w, b = x.double(), (w.double() if w is not None else 1.0), (b.double() if b is not None else 0.0)
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1 / (d.square().mean(1) + eps).sqrt()
    mean_err = 128 * EPS * x.abs().mean(1)
    assert bool(((r.mean.double() - mean).abs() <= mean_err + TINY["f32"]).all())
    assert bool(((r.rstd.double() / rstd - 1).abs() <= 70 * EPS + (mean_err * rstd).square() / 2).all())
    xh = d * rstd[:, None]
    off = (mean_err[:, None] + EPS * d.abs()) * rstd[:, None] + (72 * EPS + (mean_err * rstd).square()[:, None]) * xh.abs()
    want = xh * w + b
    bw = w.abs() if torch.is_tensor(w) else 1.0
    bb = b.abs() if torch.is_tensor(b) else 0.0
    tol = off * bw + 2 * EPS * (xh.abs() * bw + bb) + HALF[dtype] * (1 + 1e-3) * want.abs() + TINY[dtype]
    err = (r.y.double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


def _check_backward(g, dy, x, mean, rstd, w, dtype, wtype):
    n, D = x.shape
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    xh = (x - mean) * rstd
    gr = dy * (w.double() if w is not None else 1.0)
    want = rstd * (gr - gr.mean(1, keepdim=True) - xh * (gr * xh).mean(1, keepdim=True))
    tol = 140 * EPS * rstd * (gr.abs() + gr.abs().mean(1, keepdim=True) + xh.abs() * (gr * xh).abs().mean(1, keepdim=True))
    tol = tol + HALF[dtype] * (1 + 1e-3) * want.abs() + TINY[dtype]
    if g.grad_x is not None:
        err = (g.grad_x.double() - want).abs()
        assert bool((err <= tol).all()), float((err / tol).max())
    if g.grad_weight is not None:
        for got, terms in ((g.grad_weight, dy * xh), (g.grad_bias, dy)):
            want = terms.sum(0)
            tol = (min(n, 992) + 8) * EPS * terms.abs().sum(0) + HALF[wtype] * (1 + 1e-3) * want.abs() + TINY[wtype]
            err = (got.double() - want).abs()
            assert bool((err <= tol).all()), float((err / tol).max())


# Rows of one value to 8192, at and around vectors, warps and blocks; one row to many.
SHAPES = [(1, 1), (1, 100), (5, 2), (3, 3), (100, 4), (257, 7), (33, 8), (1000, 16), (4096, 100), (77, 127), (513, 128), (64, 255), (1, 256),
          (300, 257), (999, 512), (65, 513), (130, 1000), (129, 1024), (1, 2048), (700, 2048), (64, 2049), (50, 4095), (40, 4096), (33, 5001),
          (7, 8191), (330, 8192), (20_001, 33), (60_001, 10)]


@pytest.mark.parametrize("dtype, wtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("n, D", SHAPES)
def test_against_fp64(n, D, dtype, wtype):
    x, dy, w, b = _inputs(n, D, dtype, wtype, n + D, stride=(0, 3, 8)[(n + D) % 3])
    ln = _esspt().LayerNorm(n, D, dtype=TYPES[dtype], weight_dtype=TYPES[wtype])
    r = ln.forward(x, w, b)
    _check_forward(r, x, w, b, dtype)
    g = ln.backward(dy, x, r.mean, r.rstd, w)
    _check_backward(g, dy, x, r.mean, r.rstd, w, dtype, wtype)
    again = ln.backward(dy, x, r.mean, r.rstd, w, grad_x=torch.full_like(g.grad_x, math.nan))
    assert all(torch.equal(a, c) for a, c in zip(g, again))  # the same bits
    ln.close()


@pytest.mark.parametrize("D", [24, 100, 1000, 4104])
def test_without_weights_and_parts(D):
    """No weight or bias; one gradient without the other; fewer rows than the most."""
    x, dy, w, b = _inputs(50, D, "f32", "f32", D)
    ln = _esspt().LayerNorm(70, D)
    for ww, bb in ((None, None), (w, None), (None, b)):
        r = ln.forward(x, ww, bb)
        _check_forward(r, x, ww, bb, "f32")
        _check_backward(ln.backward(dy, x, r.mean, r.rstd, ww), dy, x, r.mean, r.rstd, ww, "f32", "f32")
    whole = ln.backward(dy, x, r.mean, r.rstd, w)
    only_x = ln.backward(dy, x, r.mean, r.rstd, w, need_weights=False)
    only_w = ln.backward(dy, x, r.mean, r.rstd, w, need_x=False)
    assert only_x.grad_weight is None and torch.equal(only_x.grad_x, whole.grad_x)
    assert only_w.grad_x is None and torch.equal(only_w.grad_weight, whole.grad_weight) and torch.equal(only_w.grad_bias, whole.grad_bias)
    none = ln.forward(x[:0], w, b)
    assert none.y.shape == (0, D)
    g = ln.backward(dy[:0], x[:0], none.mean, none.rstd, w)
    assert bool((g.grad_weight == 0).all()) and bool((g.grad_bias == 0).all())
    ln.close()


@pytest.mark.parametrize("D", [12, 200, 3000])
def test_gradients_against_differences(D):
    """d/dh of sum(y dy) along a direction: the formula in fp64 by central differences, the kernels' by products.  The
    differences' own error is of h^2 = 1e-8; the kernels' of 140 eps of magnitudes."""
    x, dy, w, b = _inputs(30, D, "f32", "f32", 5)
    ln = _esspt().LayerNorm(30, D)
    r = ln.forward(x, w, b)
    g = ln.backward(dy, x, r.mean, r.rstd, w)
    ln.close()
    dirs = [torch.randn_like(t).double() for t in (x, w, b)]

    def f(h):
        X, W, B = (t.double() + h * d for t, d in zip((x, w, b), dirs))
        d = X - X.mean(1, keepdim=True)
        return ((d / (d.square().mean(1, keepdim=True) + 1e-5).sqrt() * W + B) * dy.double()).sum()

    h = 1e-4
    want = (f(h) - f(-h)) / (2 * h)
    terms = [t.double() * d for t, d in zip(g, dirs)]
    got, mass = sum(t.sum() for t in terms), sum(t.abs().sum() for t in terms)
    assert abs(float(got - want)) <= 2e-5 * float(mass)


@pytest.mark.parametrize("D", [100, 1000, 4096])
def test_hard_rows(D):
    """Equal values give the bias; a far mean; huge and tiny rows; NaN and infinity spoil their own row, and the weights'
    gradients; rows of zeros."""
    g = torch.Generator("cuda").manual_seed(2)
    x = torch.randn((9, D), generator=g, device="cuda")
    x[0], x[1], x[5] = 0.1, 0.0, -1e30
    x[2] += 1e4
    x[3] *= 1e15
    x[4] *= 1e-18
    w, b = torch.randn(D, generator=g, device="cuda"), torch.randn(D, generator=g, device="cuda")
    ln = _esspt().LayerNorm(9, D)
    r = ln.forward(x, w, b)
    _check_forward(type(r)(r.y[[0, 1, 2, 3, 4, 6, 7, 8]], r.mean[[0, 1, 2, 3, 4, 6, 7, 8]], r.rstd[[0, 1, 2, 3, 4, 6, 7, 8]]),
                   x[[0, 1, 2, 3, 4, 6, 7, 8]], w, b, "f32")
    assert float((r.y[0] - b).abs().max()) <= 1e-4 and torch.equal(r.y[1], b)
    x[6, D // 2], x[7, 0] = math.nan, math.inf
    bad = ln.forward(x, w, b)
    assert bool(torch.isnan(bad.y[[6, 7]]).all()) and torch.equal(bad.y[[0, 1, 2, 3, 4, 8]], r.y[[0, 1, 2, 3, 4, 8]])
    dy = torch.randn((9, D), generator=g, device="cuda")
    clean = ln.backward(dy, torch.where(torch.isfinite(x), x, 0.0), r.mean, r.rstd, w)
    back = ln.backward(dy, x, bad.mean, bad.rstd, w)
    assert bool(torch.isnan(back.grad_x[[6, 7]]).all()) and torch.equal(back.grad_x[[0, 1, 2, 4, 8]], clean.grad_x[[0, 1, 2, 4, 8]])
    assert bool(torch.isnan(back.grad_weight).all()) and bool(torch.isfinite(back.grad_bias).all())
    ln.close()


def test_offsets_past_32_bits():
    n, D = 1_100_000, 2048
    x = torch.zeros((n, D), dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn((3, D), device="cuda").to(torch.bfloat16)
    ln = _esspt().LayerNorm(n, D, dtype=torch.bfloat16)
    r = ln.forward(x)
    _check_forward(type(r)(r.y[-4:], r.mean[-4:], r.rstd[-4:]), x[-4:], None, None, "bf16")
    g = ln.backward(x, x, r.mean, r.rstd, need_weights=False)
    _check_backward(type(g)(g.grad_x[-4:], None, None), x[-4:], x[-4:], r.mean[-4:], r.rstd[-4:], None, "bf16", "bf16")
    ln.close()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("D, shift", [(64, 1), (64, 4), (2048, 1), (101, 1)])
def test_addresses_off_the_vectors(D, shift, dtype):
    """Rows and weights that begin anywhere in memory."""
    n = 40
    buf = torch.randn(3 * n * D + 64, device="cuda").to(TYPES[dtype])
    x, dy = buf[shift:shift + n * D].view(n, D), buf[n * D + shift:2 * n * D + shift].view(n, D)
    w, b = buf[-D - 3:-3], buf[-D - 1:-1]
    ln = _esspt().LayerNorm(n, D, dtype=TYPES[dtype])
    y = torch.zeros(n * D + 8, dtype=TYPES[dtype], device="cuda")
    r = ln.forward(x, w, b, y=y[shift:shift + n * D].view(n, D))
    _check_forward(r, x, w, b, dtype)
    assert bool((y[:shift] == 0).all()) and bool((y[shift + n * D:] == 0).all())
    _check_backward(ln.backward(dy, x, r.mean, r.rstd, w), dy, x, r.mean, r.rstd, w, dtype, dtype)
    ln.close()


def test_another_stream_and_a_graph():
    side = torch.cuda.Stream()
    n, D = 300, 96
    ln = _esspt().LayerNorm(n, D, stream=side)
    x, dy, w, b = _inputs(n, D, "f32", "f32", 3)
    _check_forward(ln.forward(x, w, b), x, w, b, "f32")
    u, v = x.clone(), dy.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        r = ln.forward(u, w, b)
        g = ln.backward(v, u, r.mean, r.rstd, w)
    for X, Y in ((x, dy), (dy.contiguous(), x), (x, dy)):
        u.copy_(X), v.copy_(Y)
        graph.replay()
        _check_forward(r, u, w, b, "f32")
        _check_backward(g, v, u, r.mean, r.rstd, w, "f32", "f32")
    torch.cuda.synchronize()
    ln.close()


def test_refusals():
    e = _esspt()
    ln = e.LayerNorm(8, 4, backward=False)
    x, w = torch.zeros((8, 4), device="cuda"), torch.zeros(4, device="cuda")
    s = torch.zeros(8, device="cuda")
    for call in (
        lambda: e.LayerNorm(0, 4), lambda: e.LayerNorm(8, 9000), lambda: e.LayerNorm(8, 4, eps=0.0),
        lambda: e.LayerNorm(8, 4, weight_dtype=torch.float16), lambda: e.LayerNorm(8, 4, dtype=torch.float64),
        lambda: ln.backward(x, x, s, s, w), lambda: ln.forward(x.half(), w, w), lambda: ln.forward(x[:, :3], w, w),
        lambda: ln.forward(x, w[:3], w), lambda: ln.forward(x, w, w.half()), lambda: ln.forward(x.cpu(), w, w),
        lambda: ln.forward(torch.zeros((9, 4), device="cuda"), w, w), lambda: ln.forward(x, w, w, y=x[:7]),
    ):
        with pytest.raises(e.EssptError):
            call()
    ln.close()
    ln = e.LayerNorm(8, 4)
    for call in (lambda: ln.backward(x[:7], x, s, s, w), lambda: ln.backward(x, x, s[:7], s, w), lambda: ln.backward(x, x, s, s.half(), w)):
        with pytest.raises(e.EssptError):
            call()
    ln.close()


# Sums over a row: up to 16 additions of a thread, 5 of a warp and 4 of warps, and a product: 26, taken as 32 eps.
SUM = 32 * EPS


def _check_far_rows(r, x, w, b, dtype, eps=1e-5):
    """As _check_forward, where the mean may be far from zero.  The first mean is off by up to e1 = SUM mean|x|; differences d to
    it are at most e1 + |x - mean|, off by eps of that.  Beyond 8 standard deviations the mean is corrected by theirs, which
    is off by SUM of their greatest, so that x - mean is off by (SUM + 3 eps) times that in all (e), whatever the mean is; below, by e1
    more, and the variance by e1^2.  The sum of squares about the first mean, less D times the correction's square, is off by 3 SUM + 6 eps of D
    times the greatest d's square; 1 / sqrt by half of that, and 4 eps.  The mean that is given is one rounding more."""
    x, w, b = x.double(), w.double(), b.double()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    var = d.square().mean(1, keepdim=True) + eps
    rstd = 1 / var.sqrt()
    e1 = SUM * x.abs().mean(1, keepdim=True)
    top = d.abs().amax(1, keepdim=True) + e1
    near = torch.where(mean.abs() * rstd < 8.01, e1, 0.0)
    e = (SUM + 3 * EPS) * top + near
    rel = (1.5 * SUM + 3 * EPS) * top.square() / var + (near * rstd).square() + 4 * EPS
    assert bool(((r.mean.double()[:, None] - mean).abs() <= EPS * mean.abs() + e + TINY["f32"]).all())
    assert bool(((r.rstd.double()[:, None] / rstd - 1).abs() <= rel).all())
    xh = d * rstd
    want = xh * w + b
    tol = (e * rstd + (rel + 3 * EPS) * xh.abs()) * w.abs() * (1 + rel) + 2 * EPS * ((xh * w).abs() + b.abs())
    tol = tol + HALF[dtype] * (1 + 1e-3) * want.abs() + TINY[dtype]
    err = (r.y.double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


FAR = [1000.1, 4097.3, 20000.7, 65000.3, -1e5, 1e-5, 3e9]


def _far(dtype):
    x = torch.tensor(FAR, device="cuda")
    return (x.clamp(-40_000, 40_000) if dtype == "f16" else x).to(TYPES[dtype])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("D", [1, 7, 33, 100, 500, 513, 1000, 1002, 2049, 8192])
def test_equal_values_give_the_bias(D, dtype):
    """Whatever the value is: the sum's and the mean's roundings are taken off again, where they count."""
    x = _far(dtype)[:, None].expand(-1, D).contiguous()
    _, _, w, b = _inputs(1, D, dtype, "f32", D)
    ln = _esspt().LayerNorm(len(FAR), D, dtype=TYPES[dtype], weight_dtype=torch.float32)
    r = ln.forward(x, w, b)
    ln.close()
    _check_far_rows(r, x, w, b, dtype)
    # rstd is 1 / sqrt(eps) = 317 at most; |x^| SUM^2 |x| rstd, or SUM |x| rstd where that is below 8 SUM
    size = x[:, :1].double().abs()
    assert torch.equal(r.mean[size[:, 0] > 0.026], x[:, 0].float()[size[:, 0] > 0.026])
    tol = torch.where(size < 0.026, SUM, SUM * SUM) * size * 317 * w.double().abs() + HALF[dtype] * 1.001 * b.double().abs() + TINY[dtype]
    assert bool(((r.y.double() - b.double()).abs() <= tol).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("D", [2, 33, 100, 500, 513, 1000, 2049, 8192])
def test_rows_near_one_value(D, dtype):
    """Rows that vary by a few of their type's last places about a far mean; a part of a wide row far from the rest."""
    g = torch.Generator("cuda").manual_seed(D)
    far = _far(dtype)[:5].float()
    place = torch.exp2(torch.floor(torch.log2(far.abs()))) * 2 * HALF[dtype]
    x = far[:, None] + torch.randint(-2, 3, (5, D), generator=g, device="cuda") * place[:, None]
    x = torch.cat([x, x, x])
    x[5:10, :D // 3] *= -0.5
    x[10:] += torch.randn((5, D), generator=g, device="cuda") * 0.01 * x[10:].abs()
    x = x.to(TYPES[dtype])
    _, _, w, b = _inputs(1, D, dtype, "f32", D)
    ln = _esspt().LayerNorm(15, D, dtype=TYPES[dtype], weight_dtype=torch.float32)
    r = ln.forward(x, w, b)
    ln.close()
    _check_far_rows(r, x, w, b, dtype)


@pytest.mark.parametrize("D", [100, 500, 1000, 8192])
def test_rows_whose_squares_overflow(D):
    """x^ is 0 there and y the bias, with the mean corrected or not; infinity and NaN make the row NaN all the same."""
    g = torch.Generator("cuda").manual_seed(D)
    x = torch.randn((6, D), generator=g, device="cuda") * torch.tensor([1e20, 1e25, 1e30, 1e33, 1.0, 1.0], device="cuda")[:, None]
    x[4], x[5] = -1e30, 1e30
    x[4, 0] = -1.5e30
    b = torch.randn(D, generator=g, device="cuda")
    ln = _esspt().LayerNorm(6, D)
    r = ln.forward(x, None, b)
    assert torch.equal(r.y[:5], b.expand(5, D)) and bool((r.rstd[:5] == 0).all()) and bool(torch.isfinite(r.mean).all())
    assert torch.equal(r.y[5], b)  # (equal values)
    x[0, D - 1], x[1, 0], x[2, D // 2] = math.nan, math.inf, -math.inf
    y = ln.forward(x, None, b).y
    assert bool(torch.isnan(y[:3]).all()) and torch.equal(y[3:], r.y[3:])
    ln.close()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("D", [3, 16, 33, 100, 500, 1001, 2048])
def test_a_row_does_not_depend_on_its_neighbours(D, dtype):
    """Rows far from zero beside others, in any order: the same bits."""
    n = 200
    x, _, w, b = _inputs(n, D, dtype, "f32", D)
    x = (x.float() + 300.0 * (torch.rand((n, 1), device="cuda") < 0.3)).to(TYPES[dtype])
    ln = _esspt().LayerNorm(n, D, dtype=TYPES[dtype], weight_dtype=torch.float32)
    r = ln.forward(x, w, b)
    order = torch.randperm(n, device="cuda")
    s = ln.forward(x[order], w, b)
    ln.close()
    assert all(torch.equal(p[order], q) for p, q in zip(r, s))


def test_two_widths_from_two_threads():
    """Handles of one kind and several widths, whose rows take different amounts of shared memory, called at the same time.
    The library's own calls, which other threads' run beside: with a limit of shared memory set for each call, one in thirty failed."""
    import threading

    e = _esspt()
    call, failed, done = e.lib().esspt_norm_forward, [], []

    def work(D):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                ln = e.LayerNorm(2, D, stream=stream)
                x = torch.randn((2, D), device="cuda")
                want = ln.forward(x).y
                y = torch.zeros_like(x)
                args = (ln._h, x.data_ptr(), D, 2, None, None, y.data_ptr(), None, None)
                for _ in range(300):
                    failed.extend(D for _ in range(50) if call(*args) != e.OK)
                    stream.synchronize()
                assert torch.equal(y, want)
                ln.close()
            done.append(D)
        except Exception as err:  # noqa: BLE001
            failed.append((D, err))

    widths = (8192, 5000, 4800, 7000, 8192, 5000)
    threads = [threading.Thread(target=work, args=(D,)) for D in widths]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed and len(done) == len(widths), failed[:10]


@pytest.mark.parametrize("n, D", [(60_001, 10), (20_001, 33), (4096, 100), (3001, 1000), (700, 2048), (330, 8192)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_no_row_is_lost_from_the_sums(n, D, dtype):
    """db of whole numbers: sums below 2^24, which no order rounds."""
    g = torch.Generator("cuda").manual_seed(n)
    x = torch.randn((n, D), generator=g, device="cuda").to(TYPES[dtype])
    dy = torch.randint(-8, 9, (n, D), generator=g, device="cuda").to(TYPES[dtype])
    ln = _esspt().LayerNorm(n, D, dtype=TYPES[dtype], weight_dtype=torch.float32)
    r = ln.forward(x)
    got = ln.backward(dy, x, r.mean, r.rstd).grad_bias
    ln.close()
    assert torch.equal(got.double(), dy.double().sum(0))
