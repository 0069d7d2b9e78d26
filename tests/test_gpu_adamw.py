"""AdamW over many tensors on the GPU, against the formula.

With 32 bits against fp64, eps = 2^-24: m = b1 m + (1 - b1) g has three roundings and two rounded constants, 4 eps of its
terms' magnitudes; v one more product, 5 eps of itself; sqrt(v) 3.5 eps; the step lr/c1 m / (sqrt(v)/c2 + eps) another
16 eps of itself and m's error through the same quotient; p 3 eps; a copy half a unit more.
With 8 bits the moments' steps are single fp32 operations in a given order, so what is held is compared bit for bit with
a restatement on whole numbers (numpy).
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

EPS = 2.0**-24
B1, B2, E, LR = 0.9, 0.999, 1e-8, 1e-2


def _esspt():
    from paper_1410_8043_gb300 import esspt

    return esspt


def _flat(like, places, values, tensors):
    out = torch.zeros(values, dtype=like, device="cuda")
    for at, t in zip(places, tensors):
        out[at:at + t.numel()] = t.reshape(-1)
    return out


def _tensors(shapes, seed, std=0.1, dtype=torch.float32):
    g = torch.Generator("cuda").manual_seed(seed)
    return [(torch.randn(s, generator=g, device="cuda") * std).to(dtype) for s in shapes]


SHAPES = [(1,), (127,), (128,), (129,), (3, 5), (0,), (4096,), (4097,), (100, 100), (31, 1000), (64,), (2, 70_001)]
LISTS = {"mixed": SHAPES, "one": [(1,)], "empty": [(0,), (0, 4)], "large": [(1_000_003, 3)], "many": [(k % 7 * 30,) for k in range(1000)]}


def _step64(p, g, m, v, t, decay, lr=LR, eps=E):
    m = B1 * m + (1 - B1) * g
    v = B2 * v + (1 - B2) * g * g
    step = lr / (1 - B1**t) * m / (v.sqrt() / math.sqrt(1 - B2**t) + eps)
    return p * (1 - lr * decay) - step, m, v, step


@pytest.mark.parametrize("copy", [None, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kind", list(LISTS))
def test_32_bits_against_fp64(kind, copy):
    """Three steps from zero moments, each from the state before it; a mixed list has copies for every other tensor."""
    shapes = LISTS[kind]
    params = _tensors(shapes, 1)
    copies = [p.to(copy) if copy and (kind != "mixed" or k % 2) else None for k, p in enumerate(params)]
    decay = [0.1 * (k % 3) for k in range(len(shapes))]
    opt = _esspt().AdamW(params, copies=copies, betas=(B1, B2), eps=E, weight_decay=decay)
    for t in range(1, 4):
        grads = [g if c is None else g.to(copy) for g, c in zip(_tensors(shapes, t + 10, 0.01), copies)]
        before = opt.moments()
        m0, v0 = before.m.clone().double(), before.second.clone().double()
        p0 = [p.clone().double() for p in params]
        opt.step(grads, LR)
        after = opt.moments()
        for k, at in enumerate(opt.places):
            n = params[k].numel()
            g, m, v = grads[k].double().reshape(-1), m0[at:at + n], v0[at:at + n]
            p, m1, v1, step = _step64(p0[k].reshape(-1), g, m, v, t, decay[k])
            m_off = 4 * EPS * (B1 * m.abs() + (1 - B1) * g.abs())
            assert bool(((after.m[at:at + n] - m1).abs() <= m_off + 1e-44).all())
            assert bool(((after.second[at:at + n] - v1).abs() <= 5 * EPS * v1 + 1e-44).all())
            den = v1.sqrt() / math.sqrt(1 - B2**t) + E
            tol = 3 * EPS * p0[k].reshape(-1).abs() + EPS * p.abs() + 16 * EPS * step.abs() + LR / (1 - B1**t) * m_off / den
            assert bool(((params[k].reshape(-1) - p).abs() <= tol).all())
            if copies[k] is not None:
                assert torch.equal(copies[k], params[k].to(copy))
        inside = torch.zeros(opt.values, dtype=torch.bool, device="cuda")
        for k, at in enumerate(opt.places):
            inside[at:at + params[k].numel()] = True
        assert bool((after.m[~inside] == 0).all()) and bool((after.second[~inside] == 0).all())
    assert opt.steps == 3
    opt.close()


# -- 8 bits, restated -----------------------------------------------------------
F = np.float32


def _mix(x):
    x = ((x ^ (x >> 16)) * 0x5851F42D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x2545F491) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random(n, t, seed):
    key = _mix((seed & 0xFFFFFFFF) ^ _mix((seed >> 32) ^ _mix(t & 0xFFFFFFFF)))
    i = np.arange(n, dtype=np.uint64)
    return _mix((((i & 0xFFFFFFFF) * 0x9E3779B1 + (i >> 32) * 0x85EBCA77) & 0xFFFFFFFF) ^ key)


def _hold(x, fraction, r, keep):
    """What x (fp32, of a multiple of 128 values) is held as: by value, with whole steps d of each binade."""
    a = np.abs(x).astype(np.float64).reshape(-1, 128)
    r = r.astype(np.float64).reshape(-1, 128) / 65536
    top = a.max(1, keepdims=True)
    frac, e = np.frexp(np.where(top > 0, top, 1.0))
    e = np.where(top > 0, e - 1 + (2 * frac > 2 - 1 / fraction), -1000)
    e = np.maximum(e, -111)
    least = (1 + 1 / fraction) * 2.0 ** (e - 15)
    d = 2.0 ** (np.frexp(np.maximum(a, least))[1] - 1) / fraction
    out = np.floor(a / d + r) * d
    low = np.where(a > 0, least, 0.0) if keep else np.where(a >= (1 - r) * least, least, 0.0)
    return (np.where(a >= least, out, low) * np.sign(x.reshape(-1, 128))).reshape(-1).astype(F)


def _step8(g, m, u, t, seed):
    c = [F(B1), F(1 - B1), F(B2), F(1 - B2)]
    v = u * u
    m = m * c[0] + g * c[1]
    v = v * c[2] + (g * g) * c[3]
    h = _random(g.size, t, seed)
    u = np.sqrt(v)
    return m, u, _hold(m, 8, h >> 16, False), _hold(u, 16, h & 0xFFFF, True)


@pytest.mark.parametrize("copy", [None, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kind", ["mixed", "one", "empty", "many"])
def test_8_bits_bit_for_bit(kind, copy):
    shapes = LISTS[kind]
    seed = 0x123456789ABCDEF0
    params = _tensors(shapes, 1)
    copies = [p.to(copy) if copy and (kind != "mixed" or k % 2) else None for k, p in enumerate(params)]
    opt = _esspt().AdamW(params, copies=copies, betas=(B1, B2), eps=E, weight_decay=0.02, state_bits=8, seed=seed)
    m, u = np.zeros(opt.values, F), np.zeros(opt.values, F)
    for t in range(1, 6):
        # values from 2^-40 to 1, zeros among them
        grads = [g * torch.exp2(-40 * torch.rand_like(g)) * (torch.rand_like(g) < 0.9) for g in _tensors(shapes, t + 10, 1.0)]
        grads = [g if c is None else g.to(copy) for g, c in zip(grads, copies)]
        g = _flat(torch.float32, opt.places, opt.values, [x.float() for x in grads]).cpu().numpy()
        p0 = _flat(torch.float64, opt.places, opt.values, params)
        opt.step(grads, LR)
        m1, u1, m, u = _step8(g, m, u, t, seed)
        held = opt.moments()
        assert np.array_equal(held.m.float().cpu().numpy(), m) and np.array_equal(held.second.float().cpu().numpy(), u)
        step = LR / (1 - B1**t) * m1.astype(np.float64) / (u1.astype(np.float64) / math.sqrt(1 - B2**t) + E)
        want = p0.cpu().numpy() * (1 - LR * 0.02) - step
        got = _flat(torch.float32, opt.places, opt.values, params).cpu().numpy()
        assert (np.abs(got - want) <= 4 * EPS * np.abs(p0.cpu().numpy()) + EPS * np.abs(want) + 16 * EPS * np.abs(step)).all()
        for p, c in zip(params, copies):
            assert c is None or torch.equal(c, p.to(copy))
    opt.close()


def test_8_bits_follow_a_slow_average():
    """A constant gradient: the second moment's root grows as sqrt(1 - b2^t) |g|, held to 1/16, over 2000 steps, where
    rounding to the nearest would stand still.  The mean over 4096 values is off by few of sd 1/16 / sqrt(4096)."""
    p = torch.zeros(4096, device="cuda")
    opt = _esspt().AdamW([p], betas=(B1, B2), state_bits=8, seed=3)
    g = torch.full_like(p, 0.5)
    for _ in range(2000):
        opt.step([g], 0.0)
    u = opt.moments().second.float()
    m = opt.moments().m.float()
    assert abs(float(u.square().mean()) / (0.25 * (1 - B2**2000)) - 1) < 0.02
    assert abs(float(m.mean()) / 0.5 - 1) < 0.02
    opt.close()


def test_8_bit_codes_round_trip():
    """What `moments` gives is taken back exactly; other values go to the nearest code; extremes."""
    e = _esspt()
    p = torch.zeros(1000, device="cuda")
    opt = e.AdamW([p, p[:0]], state_bits=8)
    x = torch.randn(1024, device="cuda") * torch.exp2(torch.randint(-60, 60, (8, 1), device="cuda").float()).expand(8, 128).reshape(-1)
    x[7] = 0
    opt.load(x, x.abs(), 5)
    one = opt.moments()
    x = x.bfloat16().float()  # (what the library gets)
    x[1000:] = 0
    # half a step: 1/16 (m) and 1/32 (u) of the value, down to the least code (1 + 1/8 or 1 + 1/16) 2^(E - 15), where
    # 2^E <= 2 top of the block: below it m is off by half of that, u, which is held as it, by all of it
    top = x.abs().view(8, 128).amax(1, keepdim=True).expand(8, 128).reshape(-1)
    assert bool(((one.m.float() - x).abs() <= torch.maximum(x.abs() / 16, 1.125 * 2.0**-15 * top)).all())
    assert bool(((one.second.float() - x.abs()).abs() <= torch.maximum(x.abs() / 32, 1.0625 * 2.0**-14 * top)).all())
    opt.load(one.m.float(), one.second.double(), 5)
    two = opt.moments()
    assert torch.equal(one.m, two.m) and torch.equal(one.second, two.second) and opt.steps == 5
    # the largest of a block, at and past the last code of a binade; tiny and subnormal blocks; negative seconds
    for top in (1.875, 1.88, 1.99, 1.0, 3.0e38, 2.0**-100, 2.0**-126, 1e-40):
        y = torch.full((1024,), top, device="cuda")
        y[1::2] = -top
        opt.load(y, y, 0)
        m, u = opt.moments()
        y = y.bfloat16().float()
        least = 1.125 * 2.0**-126
        assert bool(((m[:1000].float() - y[:1000]).abs() <= y[:1000].abs().clamp(min=least) / 16 * 1.01).all() if top > least else
                    ((m[:1000].abs() == 0) | (m[:1000].abs() == least)).all())
        assert bool((u[1:1000:2] == 0).all()) and bool((u[0:1000:2] > 0).all())
    opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_absent_gradients_scale_and_rates_on_the_device(bits):
    """None leaves a tensor, its copy and moments; lr and the gradients' factor from the device."""
    e = _esspt()
    shapes = [(300,), (5000,), (77,)]
    a, b = _tensors(shapes, 1), _tensors(shapes, 1)
    one, two = (e.AdamW(x, state_bits=bits, weight_decay=0.0) for x in (a, b))
    lr, scale = torch.tensor(0.02, device="cuda"), torch.tensor([0.25], device="cuda")
    for t in range(3):
        g = _tensors(shapes, t + 3)
        g[1] = None
        one.step(g, lr, grad_scale=scale)
        two.step([None if x is None else x * 0.25 for x in g], 0.02)
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and torch.equal(a[1], _tensors(shapes, 1)[1])
    assert bool((one.moments().m[one.places[1]:one.places[2]] == 0).all()) and not torch.equal(a[0], _tensors(shapes, 1)[0])
    one.step([None] * 3, 0.1)
    assert one.steps == 4 and torch.equal(a[0], b[0])
    one.close(), two.close()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_addresses_off_the_vectors(bits, shift):
    """The same bits wherever a tensor and its gradient begin, and nothing written beside it."""
    e = _esspt()
    n = 9001
    p, g = _tensors([(n,), (n,)], 5)
    buf, gbuf, cbuf = torch.full((n + 8,), 7.0, device="cuda"), torch.zeros(n + 8, dtype=torch.float16, device="cuda"), \
        torch.full((n + 8,), 7.0, dtype=torch.float16, device="cuda")
    q, h, c = buf[shift:shift + n], gbuf[4 - shift:4 - shift + n], cbuf[shift:shift + n]
    q.copy_(p), h.copy_(g)
    p2, c2 = p.clone(), p.half()
    one = e.AdamW([q], copies=[c], state_bits=bits, seed=9)
    two = e.AdamW([p2], copies=[c2], state_bits=bits, seed=9)
    for _ in range(2):
        one.step([h], LR), two.step([g.half()], LR)
    assert torch.equal(q, p2) and torch.equal(c, c2) and torch.equal(one.moments().m, two.moments().m)
    assert bool((buf[:shift] == 7).all()) and bool((buf[shift + n:] == 7).all()) and bool((cbuf[:shift] == 7).all()) and bool((cbuf[shift + n:] == 7).all())
    one.close(), two.close()


def test_special_gradients():
    """NaN and infinity: their own value with 32 bits, and with 8 their block's moments."""
    e = _esspt()
    for bits in (32, 8):
        p = _tensors([(1000,)], 1)[0]
        opt = e.AdamW([p], state_bits=bits)
        g = _tensors([(1000,)], 2)[0]
        g[300], g[700] = math.nan, math.inf
        opt.step([g], LR)
        bad = torch.zeros(1000, dtype=torch.bool, device="cuda")
        bad[[300, 700]] = True
        assert bool(torch.isnan(p[bad]).all()) and bool(torch.isfinite(p[~bad]).all())
        opt.step([torch.zeros_like(g)], LR)
        if bits == 8:
            bad[256:384], bad[640:768] = True, True
        assert bool(torch.isnan(p[bad]).all()) and bool(torch.isfinite(p[~bad]).all())
        opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_graph_counts_its_steps(bits):
    """A step captured once and replayed is as many steps made by hand; another stream is the handle's."""
    e = _esspt()
    side = torch.cuda.Stream()
    shapes = [(1000,), (40, 41)]
    a, b = _tensors(shapes, 1), _tensors(shapes, 1)
    one, two = e.AdamW(a, state_bits=bits, stream=side), e.AdamW(b, state_bits=bits)
    grads = [torch.zeros_like(x) for x in a]
    lr = torch.tensor(LR, device="cuda")
    one.step(_tensors(shapes, 2), LR)  # by hand first
    two.step(_tensors(shapes, 2), LR)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        one.step(grads, lr)
    for t in range(4):
        for x, y in zip(grads, _tensors(shapes, t + 5)):
            x.copy_(y)
        lr.fill_(LR / (t + 1))
        graph.replay()
        two.step(_tensors(shapes, t + 5), LR / (t + 1))
    torch.cuda.synchronize()
    for x, y in zip(a, b):
        assert float((x - y).abs().max()) <= 4e-7  # (lr: a double by hand, fp32 on the device)
    assert one.steps == two.steps == 5
    one.close(), two.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_resumed_from_a_checkpoint(bits):
    """Moments and steps taken over by another handle: the same bits onwards."""
    e = _esspt()
    shapes = [(1000,), (40, 41)]
    a = _tensors(shapes, 1)
    one = e.AdamW(a, state_bits=bits, seed=4)
    for t in range(3):
        one.step(_tensors(shapes, t), LR)
    b = [x.clone() for x in a]
    two = e.AdamW(b, state_bits=bits, seed=4)
    held = one.moments()
    two.load(held.m, held.second, one.steps)
    for t in range(3):
        one.step(_tensors(shapes, t + 7), LR)
        two.step(_tensors(shapes, t + 7), LR)
    # (beta to the power t: a product of steps here, a power there)
    assert all(float((x - y).abs().max()) <= 2e-7 for x, y in zip(a, b))
    assert torch.equal(one.moments().m, two.moments().m) and torch.equal(one.moments().second, two.moments().second)
    one.close(), two.close()


def test_offsets_past_32_bits():
    n = 2**31 + 1000
    p = torch.zeros(n, device="cuda")
    opt = _esspt().AdamW([p], state_bits=8, weight_decay=0.0)
    g = torch.zeros(n, dtype=torch.float32, device="cuda")
    g[-900:] = 0.5
    opt.step([g], LR)
    assert bool((p[:-900:4097] == 0).all()) and float((p[-900:] + LR).abs().max()) <= 1e-7
    assert bool(((opt.moments().m[:n][-900:].float() - 0.05).abs() <= 0.05 / 8).all())
    opt.close()


def test_refusals():
    e = _esspt()
    p = torch.zeros((4, 6), device="cuda")
    h = p.half()
    for call in (
        lambda: e.AdamW([]), lambda: e.AdamW([h]), lambda: e.AdamW([p.T]), lambda: e.AdamW([p, p.cpu()]),
        lambda: e.AdamW([p], copies=[p]), lambda: e.AdamW([p], copies=[h[:3]]), lambda: e.AdamW([p], copies=[]),
        lambda: e.AdamW([p, p + 1], copies=[h, p.bfloat16()]), lambda: e.AdamW([p], betas=(1.0, 0.9)),
        lambda: e.AdamW([p], eps=0.0), lambda: e.AdamW([p], weight_decay=-1.0), lambda: e.AdamW([p], weight_decay=[0.0, 0.0]),
        lambda: e.AdamW([p], state_bits=16),
    ):
        with pytest.raises(e.EssptError):
            call()
    opt = e.AdamW([p], copies=[h])
    for call in (
        lambda: opt.step([], LR), lambda: opt.step([p], LR), lambda: opt.step([h.cpu()], LR), lambda: opt.step([h[:3]], LR),
        lambda: opt.step([h], math.inf), lambda: opt.step([h], torch.zeros(2, device="cuda")),
        lambda: opt.step([h], LR, grad_scale=torch.zeros(1)), lambda: opt.load(p, p, 0),
        lambda: opt.load(torch.zeros(128, device="cuda"), torch.zeros(128, device="cuda"), -1),
    ):
        with pytest.raises(e.EssptError):
            call()
    assert opt.steps == 0 and bool((p == 0).all())
    opt.close()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("lr, decay", [(1e-5, 0.01), (2e-6, 0.01), (1e-3, 0.1)])
def test_small_decay_adds_up(lr, decay, bits):
    """lr decay near 2^-23 (1e-7) and below 2^-25 (2e-8), where 1 - lr decay has one bit of it, or none.

    Two handles on the same gradients, with decay and without: their moments, and so their steps, have the same bits, and
    the mean difference of the parameters grows each step by lr decay times the mean of those that decay.  Values in (1, 2)
    lie 2^-23 apart; steps of many sizes (after the first, which is lr for all) round them either way, off by a sd of
    2^-23 / sqrt(12) each, and in the first step all by half of 2^-23 at most.  So over T steps of N values the mean is off by
    8 sd sqrt(2 T / N) + 2^-23; lr decay has two roundings, a step's sum one (2 + 1 eps of itself, taken as 8)."""
    N, T = 1 << 20, 64
    g = torch.Generator("cuda").manual_seed(7)
    p = torch.rand(N, generator=g, device="cuda") * 0.5 + 1.25
    q = p.clone()
    with_, without = _esspt().AdamW([p], state_bits=bits, weight_decay=decay, seed=5), _esspt().AdamW([q], state_bits=bits, weight_decay=0.0, seed=5)
    want = 0.0
    for _ in range(T):
        grad = torch.randn(N, generator=g, device="cuda") * 0.1
        want += lr * decay * float(p.double().mean())
        with_.step([grad], lr), without.step([grad], lr)
    assert torch.equal(with_.moments().m, without.moments().m)
    got = float((q.double() - p.double()).mean())
    tol = 8 * 2.0**-23 / math.sqrt(12) * math.sqrt(2 * T / N) + 2.0**-23 + 8 * EPS * want
    assert abs(got - want) <= tol, (got, want, tol)
    with_.close(), without.close()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("decay", [0.0, 0.1])
def test_parameters_that_are_no_numbers(bits, decay):
    """An infinite parameter stays that (p (1 - lr decay) less a step), NaN stays NaN, and neither touches another."""
    p = _tensors([(600,)], 3)[0]
    p[5], p[200], p[599] = math.inf, -math.inf, math.nan
    opt = _esspt().AdamW([p], state_bits=bits, weight_decay=decay)
    for t in range(3):
        opt.step(_tensors([(600,)], t), LR)
    assert float(p[5]) == math.inf and float(p[200]) == -math.inf and math.isnan(float(p[599]))
    assert int(torch.isfinite(p).sum()) == 597
    opt.close()


def test_the_same_tensor_twice():
    """Refused; neighbours in one buffer are not."""
    e = _esspt()
    buf = torch.zeros(1000, device="cuda")
    for params in ([buf, buf], [buf[:300], buf[299:]], [buf, buf[500:501]]):
        with pytest.raises(e.EssptError) as err:
            e.AdamW(params)
        assert err.value.status == e.EINVAL
    opt = e.AdamW([buf[300:], buf[:300], buf[:0]], weight_decay=0.0)
    opt.step([torch.ones(700, device="cuda"), torch.ones(300, device="cuda"), buf[:0]], LR)
    assert float((buf + LR).abs().max()) <= 1e-7
    opt.close()
