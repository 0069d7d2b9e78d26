"""Softmax over a catalogue on the GPU (cross entropy and distillation), against the
definition in fp64.

Tolerances, with eps = 2^-24 and sums over absolute values:
  * a score s = b h.w is a sum of D products; each product is off by at most 8 eps
    of itself (fp32 rows may be taken in two halves of 11 bits each) and each of the
    D additions by 2 eps of the sum so far (additions may truncate), so s by at most
    ds = 2 (D + 8) eps b max_v sum |h w|;
  * lse: ds, plus sums of positive terms in chains of fewer than 168 additions
    (168 eps < 1e-5), exponentials of 4 eps, and 8 eps of lse for its own arithmetic;
  * p: 2 ds + 1e-5 of itself, plus its rounding to the type that meets the tensor
    core (the type's half-unit, 2^-8 bf16, 2^-11 fp16; fp32 keeps 22 bits);
    fp16 and halves of fp32 are kept 2^14 times as large, weights at most one beside
    them, in units of 2^-24 at least: of more than eight rows p is off by at most
    2^-38 (two half-units) besides; in dh, where the largest probability may be kept as
    2^4 only, by 2^-28;
  * gradients: that times sum |terms|, plus 1e-4 of it for the additions (chains of
    at most 800 truncating ones, 2 eps each), plus the rounding of the result.
Each gradient's error is also held in its 2-norm, where rounding errors average: fp32
1e-5, bf16 2^-8, fp16 2^-11 (the half-unit of the type) of the gradient's norm.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

EPS = 2.0**-24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_UNIT = {name: torch.finfo(t).eps / 2 for name, t in TYPES.items()}
P_ROUND = {**HALF_UNIT, "f32": 2.0**-22}
TINY = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0**-24}
NORM = {"f32": 1e-5, "bf16": 2.0**-8, "f16": 2.0**-11}


def _esspt():
    from paper_1410_8043_gb300 import esspt

    return esspt


def _reference(h, w, ids, z, weight, b):
    """Definition in fp64: loss, lse, gradients, and the sums of absolute terms."""
    kept = ids >= 0
    zz = torch.where(kept, z.double() * b, -math.inf)
    live = (zz > -math.inf).any(1)
    q = torch.where(live[:, None], torch.softmax(zz, 1), 0.0).nan_to_num(0.0)
    h64 = torch.where(live[:, None], h.double(), 0.0)
    w64 = w.double()
    s = b * (h64 @ w64.T)
    lse = torch.logsumexp(s, 1)
    at = ids.long().clamp(min=0)
    logq = torch.where(q > 0, q.log(), 0.0)
    loss = torch.where(live, (q * (logq - s.gather(1, at))).sum(1) + lse * q.sum(1), 0.0)
    p = torch.exp(s - lse[:, None])
    Q = torch.zeros_like(p).scatter_add_(1, at, q)
    bw = torch.where(live, b * weight.double(), 0.0)[:, None]
    g = bw * (p - Q)
    mass = bw.abs() * (p + Q)
    return dict(
        loss=loss, lse=torch.where(live, lse, 0.0), grad_h=g @ w64, grad_w=g.T @ h64, mass_h=mass @ w64.abs(),
        mass_w=mass.T @ h64.abs(), floor_h=bw.abs() * w64.abs().sum(0), floor_w=bw.abs().max() * h64.abs().sum(0), prod=b * (h64.abs() @ w64.abs().T).amax(1), live=live, size=(zz.nan_to_num(0.0, 0.0, 0.0).abs()).amax(1),
    )


def _inputs(T, V, D, dtype, top, seed, pad=0.2, b=1.0):
    g = torch.Generator("cuda").manual_seed(seed)
    std = math.sqrt(2.0 / math.sqrt(D))
    h = (torch.randn((T, D), generator=g, device="cuda") * std).to(TYPES[dtype])
    w = (torch.randn((V, D), generator=g, device="cuda") * std).to(TYPES[dtype])
    ids = (torch.rand((T, top), generator=g, device="cuda") ** 3 * V).int().clamp_(0, V - 1)
    z = torch.randn((T, top), generator=g, device="cuda") * 2
    weight = torch.rand(T, generator=g, device="cuda") * 2 - 0.5
    drop = torch.rand((T, top), generator=g, device="cuda") < pad
    ids = ids.masked_fill(drop, -1)
    h[(ids < 0).all(1)] = math.nan
    return h, w, ids, z, weight


def _check(r, ref, dtype, D, b):
    ds = 2 * (D + 8) * EPS * ref["prod"]
    tol = ds * 2 + 1e-5 + 8 * EPS * (ref["lse"].abs() + ref["size"])
    live = ref["live"]
    for name in ("loss", "lse"):
        got = getattr(r, name).double()
        assert bool((got[~live] == 0).all()), name
        err = (got - ref[name]).abs()
        assert bool((err <= tol)[live].all()), (name, float((err / tol)[live].max()))
    if r.grad_h is None:
        return
    ep = 2 * ds + 1e-5 + P_ROUND[dtype] + 1e-4
    worst = float(ep[live].max()) if bool(live.any()) else 0.0
    for name, e in (("grad_h", ep[:, None]), ("grad_w", worst)):
        got, want, mass = getattr(r, name).double(), ref[name], ref["mass_" + name[-1]]
        err = (got - want).abs()
        bound = e * mass + HALF_UNIT[dtype] * want.abs() + TINY[dtype]
        if got.shape[0] and live.numel() > 8 and dtype != "bf16":
            bound = bound + (2.0**-28 if name == "grad_h" else 2.0**-38) * ref["floor_" + name[-1]]
        assert bool(torch.isfinite(got).all()), name
        assert bool((err <= bound).all()), (name, float((err / bound).max()))
        norm = float(want.norm())
        assert float(err.norm()) <= NORM[dtype] * norm + TINY[dtype] * math.sqrt(want.numel()), (name, float(err.norm()) / max(norm, 1e-300))


def _run(kind, h, w, ids, z, weight, b, backward=True, **kw):
    head = _esspt().SoftmaxHead(max(1, h.shape[0]), w.shape[0], w.shape[1], dtype=w.dtype, max_top=max(1, ids.shape[1]),
                                backward=backward, **kw)
    if kind == "loss":
        r = head.loss(h, w, ids[:, 0], weight=weight, inv_temperature=b)
    else:
        r = head.distill(h, w, ids, z, weight=weight, inv_temperature=b)
    head.poll()
    head.close()
    return r


# One row to many, one item to many, widths at and around the sizes of vectors,
# 16-value steps, 64-value units, 128-row tiles and the 256 columns of an accumulator.
SHAPES = [(1, 1, 1), (1, 7, 3), (3, 129, 5), (8, 1000, 16), (8, 40_001, 64), (7, 300, 512), (9, 128, 64), (16, 127, 17),
          (33, 1, 24), (97, 1000, 16), (128, 256, 64), (129, 257, 65), (130, 2050, 100), (257, 640, 33), (300, 3001, 128),
          (255, 1500, 129), (500, 2049, 192), (200, 900, 256), (129, 1100, 257), (260, 1300, 320), (140, 1000, 449),
          (300, 5000, 512), (1500, 700, 64), (2000, 4000, 48), (700, 20_000, 100)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D", SHAPES)
def test_loss_shapes(T, V, D, dtype):
    h, w, ids, z, weight = _inputs(T, V, D, dtype, 1, T + V + D)
    ref = _reference(h, w, ids, torch.zeros_like(z), weight, 1.0)
    _check(_run("loss", h, w, ids, z, weight, 1.0), ref, dtype, D, 1.0)
    _check(_run("loss", h, w, ids, z, weight, 1.0, backward=False), ref, dtype, D, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D,top", [(1, 1, 1, 1), (2, 50, 8, 3), (8, 3000, 100, 40), (8, 20_000, 64, 200), (9, 300, 7, 33),
                                       (100, 1000, 16, 8), (260, 2000, 64, 64), (700, 900, 100, 32), (300, 3000, 256, 17),
                                       (150, 2500, 512, 5), (1500, 333, 64, 31)])
def test_distill_shapes(T, V, D, top, dtype):
    h, w, ids, z, weight = _inputs(T, V, D, dtype, top, T + V + D + top)
    ref = _reference(h, w, ids, z, weight, 0.5)
    _check(_run("distill", h, w, ids, z, weight, 0.5), ref, dtype, D, 0.5)
    _check(_run("distill", h, w, ids, z, weight, 0.5, backward=False), ref, dtype, D, 0.5)


# Streams of many tiles per block: rings of stages and buffers go round several times.
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,D", [(300, 150_001, 40), (2000, 60_000, 100), (9000, 3000, 60), (400, 90_000, 150), (300, 60_001, 250),
                                   (300, 60_000, 300), (5000, 4000, 510), (1500, 50_000, 20), (1000, 70_000, 130),
                                   (1200, 61_000, 300)])
def test_long_streams(T, V, D, dtype):
    h, w, ids, z, weight = _inputs(T, V, D, dtype, 2, T + V + D)
    ref = _reference(h, w, ids, z, weight, 1.0)
    _check(_run("distill", h, w, ids, z, weight, 1.0), ref, dtype, D, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,D,top", [(1, 200_003, 24, 1), (1, 200_003, 61, 3), (1, 90_001, 500, 9), (5, 200_003, 24, 9),
                                       (5, 160_001, 61, 3), (2, 300_000, 130, 40)])
def test_few_rows_over_many_items(T, V, D, top, dtype):
    """Lists short and long, scores kept and not, widths read by vectors and by single values."""
    h, w, ids, z, weight = _inputs(T, V, D, dtype, top, T + V + D, pad=0.0 if T == 1 else 0.2)
    ref = _reference(h, w, ids, z, weight, 1.0)
    _check(_run("distill", h, w, ids, z, weight, 1.0), ref, dtype, D, 1.0)
    _check(_run("distill", h, w, ids, z, weight, 1.0, backward=False), ref, dtype, D, 1.0)
    ids[:, 0], h = V - 1, h.nan_to_num(0.0)
    ref = _reference(h, w, ids[:, :1], torch.zeros_like(z[:, :1]), weight, 1.0)
    _check(_run("loss", h, w, ids, z, weight, 1.0, backward=False), ref, dtype, D, 1.0)
    w[V // 2, D - 1] = math.nan
    assert bool(_run("loss", h, w, ids, z, weight, 1.0, backward=False).loss.isnan().all())
    r = _run("loss", h, w, ids.fill_(-1), z, weight, 1.0, backward=False)
    assert bool((r.loss == 0).all()) and bool((r.lse == 0).all())


SIDES = [(8, 700, 32), (200, 700, 32)]  # a few rows, and more


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,D", SIDES)
def test_rows_left_empty(T, V, D, dtype):
    """Every row ignored: zeros, whatever h holds; and one row kept among them."""
    h, w, ids, z, weight = _inputs(T, V, D, dtype, 4, 5)
    h.fill_(math.inf)
    ids.fill_(-1)
    for kind in ("loss", "distill"):
        r = _run(kind, h, w, ids, z, weight, 1.0)
        assert all(bool((x == 0).all()) for x in r)
    h[T // 2] = 0.5
    ids[T // 2, 0] = V - 1
    for kind in ("loss", "distill"):
        ref = _reference(h, w, ids[:, :1], torch.zeros_like(z[:, :1]), weight, 1.0)
        _check(_run(kind, h, w, ids, z, weight, 1.0), ref, dtype, D, 1.0)


@pytest.mark.parametrize("T,V,D", SIDES)
def test_teacher_lists(T, V, D):
    """Logits of -infinity, rows with nothing else, items named twice, one item for all."""
    h, w, ids, z, weight = _inputs(T, V, D, "f32", 6, 9, pad=0.0)
    z[:, 1] = -math.inf
    z[1] = -math.inf
    ids[2] = 3
    ids[3:, 2] = 17
    z[5] = 3e38  # (equal and huge: q = 1/6 each)
    ref = _reference(h, w, ids, z, weight, 0.25)
    _check(_run("distill", h, w, ids, z, weight, 0.25), ref, "f32", D, 0.25)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_popular_target(dtype):
    """One item is nearly every row's target, so its gradient sums thousands of rows."""
    T, V, D = 3000, 500, 40
    h, w, ids, z, weight = _inputs(T, V, D, dtype, 1, 3)
    ids[torch.arange(T, device="cuda") % 7 > 0] = 130
    h = h.nan_to_num(0.25)
    ref = _reference(h, w, ids, torch.zeros_like(z), weight, 1.0)
    _check(_run("loss", h, w, ids, z, weight, 1.0), ref, dtype, D, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows", [1, 700])
def test_scores_far_above_the_first_items(rows, dtype):
    """Large problems take a row's reference from its targets and W's first items.  Here
    the largest scores of some rows are of other items, 30 to 300 above: the sums leave
    the range of 16 bits (of fp32, of bf16 rows) and the call has to notice."""
    T, V, D = 1600, 50_000, 32
    h, w, ids, z, weight = _inputs(T, V, D, dtype, 3, 77, pad=0.0)
    ids = ids % 40_000
    far = torch.zeros(D, device="cuda")
    far[5] = 300.0 if dtype == "bf16" else 30.0
    h[:, 5] = 0.0
    h[100:100 + rows, 5] = 1.0
    w[49_000:49_004] = (far * torch.tensor([[0.9], [1.0], [0.99], [0.5]], device="cuda")).to(w.dtype)
    ref = _reference(h, w, ids, z, weight, 1.0)
    _check(_run("distill", h, w, ids, z, weight, 1.0), ref, dtype, D, 1.0)
    ref = _reference(h, w, ids[:, :1], torch.zeros_like(z[:, :1]), weight, 1.0)
    _check(_run("loss", h, w, ids, z, weight, 1.0), ref, dtype, D, 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T", [8, 60, 900])
def test_near_a_fit(T, dtype):
    """Targets with p of about 0.99: the gradients are the small differences p - q.  The
    other items' p keep the type's relative precision, so do the results; p of the target
    rounded to the type would be off by up to 2^-9 of one, a fifth of 1 - p and more."""
    V, D = 2000, 64
    h, w, ids, z, weight = _inputs(T, V, D, dtype, 1, 19, pad=0.0)
    weight = weight.abs() + 0.5
    h = (w[ids[:, 0].long()].float() * 0.9).to(h.dtype)
    ref = _reference(h, w, ids, torch.zeros_like(z), weight, 1.0)
    assert 1e-4 < float(ref["loss"].median()) < 5e-2
    r = _run("loss", h, w, ids, z, weight, 1.0)
    for name in ("grad_h", "grad_w"):
        err = (getattr(r, name).double() - ref[name]).norm() / ref[name].norm()
        assert float(err) <= 2 * HALF_UNIT[dtype], (name, float(err))


@pytest.mark.parametrize("T,V,D", SIDES)
@pytest.mark.parametrize("size", [1e-12, 1e-3, 30.0, 3000.0])
def test_magnitudes(T, V, D, size):
    """Scores from nothing to thousands (one item takes all), all far below or above zero."""
    h, w, ids, z, weight = _inputs(T, V, D, "f32", 1, 11)
    for shift in (0.0, -1.0, 1.0):
        w2 = w.clone()
        w2[:, 0] += 4.0 * shift
        h2 = h * size
        h2[:, 0] = h2[:, 0].abs()
        ref = _reference(h2, w2, ids, torch.zeros_like(z), weight, 1.0)
        if float(ref["prod"].max()) * 2 * (D + 8) * EPS < 0.05:  # else p itself is not determined
            _check(_run("loss", h2, w2, ids, z, weight, 1.0), ref, "f32", D, 1.0)
        else:
            r = _run("loss", h2, w2, ids, z, weight, 1.0)
            live = ref["live"]
            tol = 4 * (D + 8) * EPS * ref["prod"] + 1e-4
            assert bool(((r.loss - ref["loss"]).abs() <= tol)[live].all())
            assert all(bool(torch.isfinite(x).all()) for x in r)


def test_scales_of_h_and_w_apart():
    """Rows of 1e-20 against items of 1e20, and both small: fp32 rows of any size."""
    for T in (8, 150):
        h, w, ids, z, weight = _inputs(T, 300, 20, "f32", 1, 12)
        for a, c in ((1e-20, 1e20), (1e15, 1e-15), (1e-10, 1e-10)):
            ref = _reference(h * a, w * c, ids, torch.zeros_like(z), weight, 1.0)
            r = _run("loss", h * a, w * c, ids, z, weight, 1.0)
            tol = 4 * 28 * EPS * ref["prod"] + 1e-5 + 1e-6 * ref["lse"].abs()
            assert bool(((r.lse - ref["lse"]).abs() <= tol).all())
            for name in ("grad_h", "grad_w"):
                err = (getattr(r, name).double() - ref[name]).norm()
                assert float(err) <= 1e-5 * float(ref[name].norm()), (name, a, c)


@pytest.mark.parametrize("T,V,D", SIDES)
def test_nan_and_infinity_stay_where_they_are(T, V, D):
    """A kept row with NaN spoils its own loss and dh, and dw; no other row's loss or dh."""
    h, w, ids, z, weight = _inputs(T, V, D, "f32", 1, 13, pad=0.0)
    clean = _run("loss", h, w, ids, z, weight, 1.0)
    h[3, 1] = math.nan
    r = _run("loss", h, w, ids, z, weight, 1.0)
    others = torch.arange(T, device="cuda") != 3
    assert bool(r.loss[3].isnan()) and bool(r.grad_h[3].isnan().all()) and bool(r.grad_w.isnan().any())
    torch.testing.assert_close(r.loss[others], clean.loss[others], rtol=1e-6, atol=1e-5)
    torch.testing.assert_close(r.grad_h[others], clean.grad_h[others], rtol=1e-4, atol=1e-5)
    h, w, ids, z, weight = _inputs(T, V, D, "f32", 1, 13, pad=0.0)
    w[V - 1, D - 1] = math.nan
    assert bool(_run("loss", h, w, ids, z, weight, 1.0).loss.isnan().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [5, 140])
@pytest.mark.parametrize("gap,offset", [(0, 1), (1, 0), (3, 5), (8, 8), (60, 4)])
def test_strides_and_alignment(T, dtype, gap, offset):
    """Rows out of a wider buffer that starts anywhere; other layouts are copied."""
    V, D = 600, 40
    h, w, ids, z, weight = _inputs(T, V, D, dtype, 3, 21)
    ref = _reference(h, w, ids, z, weight, 1.0)

    def apart(x):
        buf = torch.full((x.shape[0] * (D + gap) + offset,), math.nan, device="cuda", dtype=x.dtype)
        y = buf[offset:].view(x.shape[0], D + gap)[:, :D]
        y.copy_(x)
        return y

    _check(_run("distill", apart(h), apart(w), ids, z, weight, 1.0), ref, dtype, D, 1.0)
    if gap == 0:
        _check(_run("distill", h.T.contiguous().T, w.T.contiguous().T, ids.long(), z, weight, 1.0), ref, dtype, D, 1.0)


@pytest.mark.parametrize("T,V,D", SIDES)
def test_gradients_against_differences(T, V, D):
    """d loss / d h and d w along random directions, by central differences of the fp64
    definition at a step whose error (its cube's term and cancellation) is below 1e-7."""
    h, w, ids, z, weight = _inputs(T, V, D, "f32", 4, 31, pad=0.0)
    r = _run("distill", h, w, ids, z, weight, 0.7)
    g = torch.Generator("cuda").manual_seed(1)
    for name, x in (("grad_h", h), ("grad_w", w)):
        dx = torch.randn(x.shape, generator=g, device="cuda", dtype=torch.float64)
        step, total = 1e-5, []
        for sign in (1, -1):
            moved = x.double() + sign * step * dx
            ref = _reference(moved if x is h else h.double(), moved if x is w else w.double(), ids, z, weight, 0.7)
            total.append(float((ref["loss"] * weight.double()).sum()))
        want = (total[0] - total[1]) / (2 * step)
        got = float((getattr(r, name).double() * dx).sum())
        scale = float((getattr(r, name).double().abs() * dx.abs()).sum())
        assert abs(got - want) <= 1e-5 * scale, name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,D,top", [(8, 3000, 64, 9), (1200, 900, 64, 40), (300, 2000, 300, 5)])
def test_same_bits_twice(T, V, D, top, dtype):
    h, w, ids, z, weight = _inputs(T, V, D, dtype, top, 41)
    a, b = (_run("distill", h, w, ids, z, weight, 1.0) for _ in range(2))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_calls_of_every_size_on_one_handle():
    """One handle, calls that shrink and grow, both operators, with and without gradients:
    nothing of a call is left in the next."""
    V, D = 1000, 64
    head = _esspt().SoftmaxHead(600, V, D, max_top=5)
    for T, kind, backward in [(600, "loss", True), (3, "distill", True), (130, "distill", False), (0, "loss", True),
                              (9, "loss", True), (600, "distill", True), (8, "loss", False)]:
        h, w, ids, z, weight = _inputs(T, V, D, "f32", 5, 50 + T)
        if kind == "loss":
            r = head.loss(h, w, ids[:, 0], weight=weight, backward=backward)
        else:
            r = head.distill(h, w, ids, z, weight=weight, backward=backward)
        assert (r.grad_w is not None) == backward
        if T == 0:
            assert r.loss.shape == (0,) and bool((r.grad_w == 0).all())
            continue
        if kind == "loss":
            ids, z = ids[:, :1], torch.zeros_like(z[:, :1])
        _check(r, _reference(h, w, ids, z, weight, 1.0), "f32", D, 1.0)
    r = head.loss(h, w, ids[:, 0])  # no weights: one each
    _check(r, _reference(h, w, ids, z, torch.ones(8, device="cuda"), 1.0), "f32", D, 1.0)
    head.poll()


@pytest.mark.parametrize("T", [4, 300])
def test_another_stream(T):
    """Inputs made on the current stream, a handle on another, outputs used at once."""
    V, D = 5000, 64
    side = torch.cuda.Stream()
    head = _esspt().SoftmaxHead(T, V, D, stream=side)
    for seed in range(5):
        torch.cuda._sleep(2_000_000)
        h, w, ids, z, weight = _inputs(T, V, D, "f32", 1, seed)
        r = head.loss(h, w, ids[:, 0], weight=weight)
        kept = [x.clone() for x in r]
        ref = _reference(h, w, ids, torch.zeros_like(z), weight, 1.0)
        h.fill_(math.nan), w.fill_(math.nan)
        _check(_esspt().SoftmaxResult(*kept), ref, "f32", D, 1.0)
    head.poll()


@pytest.mark.parametrize("T,V", [(6, 5000), (100, 700), (200, 5000)])
def test_captured_in_a_graph(T, V):
    """Calls of a handle on the captured stream, replayed on other values: what a call gives."""
    D = 48
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        head = _esspt().SoftmaxHead(T, V, D, max_top=3)
        h, w, ids, z, weight = _inputs(T, V, D, "f32", 3, 71)

        def both():
            return [*head.loss(h, w, ids[:, 0], weight=weight), *head.distill(h, w, ids, z, weight=weight)]

        both()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = both()
        for seed in (72, 73):
            for x, y in zip((h, w, ids, z, weight), _inputs(T, V, D, "f32", 3, seed)):
                x.copy_(y)
            graph.replay()
            got = [x.clone() for x in out]
            assert all(torch.equal(x, y) for x, y in zip(got, both()))
        head.poll()
    torch.cuda.current_stream().wait_stream(stream)


@pytest.mark.parametrize("T", [6, 200])
def test_ids_outside_the_catalogue(T):
    """They count as absent, and poll reports them once."""
    e = _esspt()
    V, D = 300, 16
    h, w, ids, z, weight = _inputs(T, V, D, "f32", 3, 61)
    outside = ids.clone()
    outside[2, :] = V
    outside[3, 1] = 2**31 - 1
    for kind in ("loss", "distill"):
        head = e.SoftmaxHead(T, V, D, max_top=3)
        cols = slice(0, 1) if kind == "loss" else slice(0, 3)
        zz = torch.zeros_like(z[:, cols]) if kind == "loss" else z
        if kind == "loss":
            r = head.loss(h, w, outside[:, 0], weight=weight)
        else:
            r = head.distill(h, w, outside, z, weight=weight)
        _check(r, _reference(h, w, outside[:, cols].masked_fill(outside[:, cols] >= V, -1), zz, weight, 1.0), "f32", D, 1.0)
        with pytest.raises(e.EssptError) as err:
            head.poll()
        assert err.value.status == e.EINVAL
        head.poll()
        head.close()


def test_refusals():
    e = _esspt()
    for bad in (dict(max_rows=0), dict(n_items=0), dict(width=0), dict(width=513), dict(max_top=0), dict(max_rows=1 << 25),
                dict(max_rows=1 << 20, max_top=1 << 11), dict(dtype=torch.float64), dict(n_items=(1 << 30) + 1)):
        with pytest.raises(e.EssptError) as err:
            e.SoftmaxHead(**{**dict(max_rows=4, n_items=10, width=8), **bad})
        assert err.value.status == e.EINVAL
    head = e.SoftmaxHead(4, 10, 8, max_top=2)
    h, w = torch.zeros(4, 8, device="cuda"), torch.zeros(10, 8, device="cuda")
    y, z = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    ids = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    head.loss(h, w, y)
    refused = [
        lambda: head.loss(h.double(), w, y), lambda: head.loss(h, w.bfloat16(), y), lambda: head.loss(h.cpu(), w, y),
        lambda: head.loss(h[:, :7], w, y), lambda: head.loss(h, w[:9], y), lambda: head.loss(h, w, y[:3]),
        lambda: head.loss(h, w, y.float()), lambda: head.loss(h, w, y, weight=torch.ones(3, device="cuda")),
        lambda: head.loss(torch.zeros(5, 8, device="cuda"), w, torch.zeros(5, dtype=torch.int32, device="cuda")),
        lambda: head.loss(h, w, y, inv_temperature=0.0), lambda: head.loss(h, w, y, inv_temperature=math.nan),
        lambda: head.loss(h, w, y, inv_temperature=math.inf), lambda: head.loss(h, w, y, grad_w=torch.zeros(9, 8, device="cuda")),
        lambda: head.distill(h, w, ids, z[:3]), lambda: head.distill(h, w, y, z), lambda: head.distill(h, w, ids, z.int()),
        lambda: head.distill(h, w, torch.zeros(4, 3, dtype=torch.int32, device="cuda"), torch.zeros(4, 3, device="cuda")),
        lambda: head.distill(h, w, ids[:, :0], z[:, :0]),
    ]
    for call in refused:
        with pytest.raises(e.EssptError) as err:
            call()
        assert err.value.status == e.EINVAL
    forward = e.SoftmaxHead(4, 10, 8, backward=False)
    assert forward.loss(h, w, y).grad_h is None
    with pytest.raises(e.EssptError):
        forward.loss(h, w, y, backward=True)


def test_c_refusals_name_their_reason():
    """The C entries check what the binding cannot get wrong."""
    import ctypes

    e = _esspt()
    L = e.lib()
    head = e.SoftmaxHead(4, 10, 8)
    cfg = e.SoftmaxConfig(4, 10, 8, 0, 1, 1, None)
    out = ctypes.c_void_p()
    ws = head.workspace
    for args, status in (((None, ws.data_ptr(), ws.numel()), e.EINVAL), ((ctypes.byref(cfg), None, ws.numel()), e.EINVAL),
                         ((ctypes.byref(cfg), ws.data_ptr() + 8, ws.numel()), e.EINVAL),
                         ((ctypes.byref(cfg), ws.data_ptr(), ws.numel() - 1), e.ENOSPC)):
        assert L.esspt_softmax_create(*args, ctypes.byref(out)) == status
        assert L.esspt_softmax_last_error(None) != b""
    h = torch.zeros(4, 8, device="cuda")
    w = torch.zeros(10, 8, device="cuda")
    y = torch.zeros(4, dtype=torch.int32, device="cuda")
    o = torch.zeros(4, device="cuda")
    gw, gh = torch.zeros_like(w), torch.zeros_like(h)
    good = [head._h, h.data_ptr(), 8, w.data_ptr(), 8, y.data_ptr(), 4, None, 1.0, o.data_ptr(), o.data_ptr(), None, None]
    assert L.esspt_softmax_loss(*good) == e.OK
    for at, value in ((1, None), (3, None), (5, None), (9, None), (10, None), (2, 7), (4, 7), (6, 5), (6, -1), (1, h.data_ptr() + 2),
                      (11, gh.data_ptr()), (12, gw.data_ptr())):
        args = list(good)
        args[at] = value
        assert L.esspt_softmax_loss(*args) == e.EINVAL, at
        assert L.esspt_softmax_last_error(head._h) != b""
    assert L.esspt_softmax_loss(None, *good[1:]) == e.EINVAL
    assert L.esspt_softmax_poll(None) == e.EINVAL and L.esspt_softmax_destroy(None) == e.OK


@pytest.mark.parametrize("T", [2, 12])
def test_catalogue_past_32_bits(T):
    """More than 2^32 values in W and its gradient; checked at rows on both sides of 2^31
    and 2^32, against the same definition by pieces."""
    V, D = 8_500_003, 512
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    w = torch.empty((V, D), device="cuda", dtype=torch.bfloat16)
    g = torch.Generator("cuda").manual_seed(7)
    for a in range(0, V, 1_000_000):
        w[a:a + 1_000_000].normal_(0.0, 0.3, generator=g)
    h = torch.randn((T, D), generator=g, device="cuda").mul_(0.3).bfloat16()
    y = torch.tensor([V - 1, 2**31 // D] * (T // 2), device="cuda", dtype=torch.int32)
    head = _esspt().SoftmaxHead(T, V, D, dtype=torch.bfloat16)
    r = head.loss(h, w, y)
    s = torch.cat([h.double() @ w[a:a + 500_000].double().T for a in range(0, V, 500_000)], 1)
    lse = torch.logsumexp(s, 1)
    assert float((r.lse - lse).abs().max()) < 1e-3
    assert float((r.loss - (lse - s.gather(1, y.long()[:, None])[:, 0])).abs().max()) < 1e-3
    rows = torch.tensor([0, 2**31 // D - 1, 2**31 // D, 2**31 // D + 1, 2**32 // D, 2**32 // D + 1, V - 2, V - 1], device="cuda")
    p = torch.exp(s[:, rows] - lse[:, None]) - (y[:, None] == rows[None]).double()
    want = p.T @ h.double()
    err = (r.grad_w[rows].double() - want).abs()
    assert bool((err <= 2.0**-7 * (p.abs().T @ h.double().abs())).all())
    gh = torch.zeros((T, D), device="cuda", dtype=torch.float64)
    for a in range(0, V, 500_000):
        part = torch.exp(s[:, a:a + 500_000] - lse[:, None])
        gh += part @ w[a:a + 500_000].double()
    gh -= w[y.long()].double()
    assert float((r.grad_h.double() - gh).norm()) <= 2.0**-7 * float(gh.norm())
