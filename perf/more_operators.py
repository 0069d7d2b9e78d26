"""What stands around the softmax over a catalogue in a training step: rows looked up, normed, and updated.

  lookup      out_t = s E[id_t]; an id < 0 is padding and gives zeros
  embed_grad  dE_v = s sum_{t: id_t = v} dout_t, over all rows of E, or added to a gradient that is there (the
              softmax's, where a catalogue's rows are inputs too); the dout of padding is not read
  norm        layer norm: x^ = (x - mean) r, r = 1 / sqrt(var + eps), y = x^ w + b.  With `train` the gradients too:
              with g = dy w, dx = r (g - mean g - x^ mean(g x^)), dw = sum_t dy x^, db = sum_t dy
  adamw       one step over a list of fp32 tensors, t the step's number:
                m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2
                p = p (1 - lr decay) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
              and, where the model runs on 16-bit copies, gradients of that type and new copies

Moments are held in 32 bits, or in 8: m and u = sqrt(v) in blocks of 128 values with an exponent E each,

  |m| = (1 + j/8) 2^(E - 15 + e),   u = (1 + j/16) 2^(E - 15 + e),   e = 0..15  (code 16 e + j or 8 e + j; code 0 is zero)

E the least (-111 at least) that the block's largest value needs.  A value x between two steps d apart is held as
d floor(x / d + rho), rho in [0, 1) a hash of the seed, the step and the value's place: moving averages of 0.999 would
stand still if they were rounded to the nearest.  Below the least code m is held as it or as zero, u as it.

Every tensor's part of a flat buffer begins at a multiple of 128 values.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
B1, B2, EPS, LR, DECAY, SEED = 0.9, 0.999, 1e-8, 1e-3, 0.01, 1410
NORM_EPS = 1e-5
M32 = 0xFFFFFFFF


def _lookup(name, T, V, D, dtype, scale=1.0, pad=0.1):
    c = dict(kind="lookup", T=T, V=V, D=D, dtype=dtype, scale=scale, pad=pad)
    return dict(c, name=name) if name else c


def _embed_grad(name, T, V, D, dtype, scale=1.0, pad=0.1, add=False):
    c = dict(kind="embed_grad", T=T, V=V, D=D, dtype=dtype, scale=scale, pad=pad, add=add)
    return dict(c, name=name) if name else c


def _norm(name, T, D, dtype, train, wtype="f32", stride=0):
    """wtype: the weights' type; stride: values between the end of a row of x and the next one's start."""
    c = dict(kind="norm", T=T, D=D, dtype=dtype, train=train, wtype=wtype, stride=stride)
    return dict(c, name=name) if name else c


def _adamw(name, tables, rows, width, vectors, bits, copy=None):
    """`tables` tensors of width `width`, the k-th of rows // (k % 3 + 1) + k rows, and `vectors` of `width` values."""
    c = dict(kind="adamw", tables=tables, rows=rows, width=width, vectors=vectors, bits=bits, copy=copy)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One item's row of the mid catalogue (18k items, rank 100): latency.
        _lookup("lookup_one_row", 1, 18_000, 100, "f32", pad=0.0),
        # The events of a batch over the largest catalogue (1M items, rank 64), scaled as inputs of a network are.
        _lookup("lookup_large", 262_147, 1_000_000, 64, "f32", scale=8.0),
        # A step on the tiny workload's 1000 items, rank 16.
        _embed_grad("embed_grad_tiny", 97, 1000, 16, "f32"),
        # Inputs and softmax share the mid catalogue: added to the softmax's gradient.
        _embed_grad("embed_grad_shared_mid", 8195, 18_000, 100, "f32", scale=10.0, add=True),
        # Half precision, sequences of a vocabulary of 50k, width 256.
        _embed_grad("embed_grad_bf16", 65_537, 50_021, 256, "bf16", scale=16.0),
        # Many events over the largest catalogue; popular items have tens of thousands of them.
        _embed_grad("embed_grad_large", 1_000_003, 1_000_000, 64, "f32"),
        # One user's row before its scores are taken: latency.
        _norm("norm_one_row", 1, 100, "f32", False),
        # A step on the mid workload's rows.
        _norm("norm_train_mid", 4096, 100, "f32", True),
        # Hidden states of a wide network, half precision, weights held in fp32.
        _norm("norm_train_wide_bf16", 32_771, 2048, "bf16", True),
        # The tiny workload's tables and a norm's vectors.
        _adamw("adamw_tiny", 2, 2000, 16, 2, 32),
        # A network's 48 matrices and 50 vectors, run in bf16 from fp32 masters.
        _adamw("adamw_many_bf16", 48, 2048, 512, 50, 32, copy="bf16"),
        # Tables of millions of rows, moments in 8 bits, read back as a checkpoint does.
        _adamw("adamw_large_8bit", 2, 2_000_000, 64, 2, 8),
    ]


def draw(rng):
    def logu(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["lookup", "embed_grad", "norm", "adamw"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if kind == "norm":
        T, D = logu(1, 300_000), logu(8, 8192)
        return _norm(None, min(T, 64_000_000 // D), D, dtype, rng.random() < 0.75, rng.choice(["f32", dtype]),
                     rng.choice([0, 0, 8, 3]))
    if kind == "adamw":
        tables, width, total = logu(1, 60), logu(8, 1024), logu(2_000, 150_000_000)
        return _adamw(None, tables, max(1, total // (tables * width)), width, logu(1, 60), rng.choice([32, 8]),
                      rng.choice([None, "bf16", "f16"]))
    T, V, D = logu(1, 1_000_000), logu(500, 1_000_000), logu(8, 1024)
    T, V = min(T, 64_000_000 // D), min(V, 64_000_000 // D)
    scale, pad = rng.choice([1.0, math.sqrt(D)]), rng.choice([0.0, 0.1, 0.5])
    if kind == "lookup":
        return _lookup(None, T, V, D, dtype, scale, pad)
    return _embed_grad(None, T, V, D, dtype, scale, pad, rng.random() < 0.3)


# -- inputs -------------------------------------------------------------------
def _randn(g, shape, std=1.0, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)


def _items(g, n, V):
    """Item ids, the k-th most popular with a share of about 1/k; ranks scattered over the ids."""
    rank = torch.rand(n, generator=g, device="cuda", dtype=torch.float64).mul_(math.log(V)).exp_().long() - 1
    return torch.randperm(V, generator=g, device="cuda")[rank.clamp_(0, V - 1)].to(torch.int32)


def _layout(case):
    """The tensors' shapes, where each begins in the flat buffers, and their length."""
    c = case
    shapes = [(c["rows"] // (k % 3 + 1) + k, c["width"]) for k in range(c["tables"])] + [(c["width"],)] * c["vectors"]
    at, end = [], 0
    for s in shapes:
        at.append(end)
        end += -(-math.prod(s) // 128) * 128
    return shapes, at, end


def _views(flat, shapes, at):
    return [flat[o:o + math.prod(s)].view(s) for s, o in zip(shapes, at)]


def _within(case):
    """Which values of the flat buffers belong to a tensor."""
    shapes, at, end = _layout(case)
    m = torch.zeros(end, dtype=torch.bool, device="cuda")
    for x in _views(m, shapes, at):
        x.fill_(True)
    return m


def prepare(case, seed):
    c = case
    g = torch.Generator("cuda")
    g.manual_seed(seed)
    s = dict(case=c)
    if c["kind"] in ("lookup", "embed_grad"):
        dtype = TYPES[c["dtype"]]
        s["ids"] = _items(g, c["T"], c["V"])
        pad = torch.rand(c["T"], generator=g, device="cuda") < c["pad"]
        s["ids"].masked_fill_(pad, -1)
        if c["kind"] == "lookup":
            s["w"] = _randn(g, (c["V"], c["D"]), c["D"] ** -0.5, dtype)
        else:
            s["grad"] = _randn(g, (c["T"], c["D"]), 1.0, dtype)
            s["grad"][pad] = math.nan
            if c["add"]:
                s["grad_w"] = _randn(g, (c["V"], c["D"]), 1.0, dtype)
    elif c["kind"] == "norm":
        dtype, wtype = TYPES[c["dtype"]], TYPES[c["wtype"]]
        x = _randn(g, (c["T"], c["D"] + c["stride"])).add_(_randn(g, (c["T"], 1), 2.0))
        x[torch.rand(c["T"], generator=g, device="cuda") < 0.05] = 0.0  # looked up for padding
        s["x"] = x.to(dtype)[:, :c["D"]]
        s["weight"], s["bias"] = (1.0 + _randn(g, c["D"], 0.1)).to(wtype), _randn(g, c["D"], 0.1, wtype)
        if c["train"]:
            s["dy"] = _randn(g, (c["T"], c["D"]), 1.0, dtype)
    else:
        shapes, at, end = _layout(c)
        dtype = TYPES[c["copy"] or "f32"]
        within = _within(c)
        s["p"] = _randn(g, end, 0.05).mul_(within)
        s["grad"] = _randn(g, end, 0.01).mul_(within).to(dtype)
        s["copy"] = s["p"].to(dtype) if c["copy"] else None
        s["t"] = 100
        if c["bits"] == 32:
            s["m"] = _randn(g, end, 0.003).mul_(within)
            s["v"] = _randn(g, end, 0.01).square_().mul_(within)
        else:  # codes as a run has left them: exponents of gradients of 1e-2, values over seven binades
            for name, top in (("m", 118), ("u", 120)):
                code = torch.randint(64 if name == "m" else 128, 127 if name == "m" else 255, (end,), generator=g, device="cuda")
                s[name] = code.mul_(within).to(torch.uint8)
                s[name + "_exp"] = torch.full((end // 128,), top, dtype=torch.uint8, device="cuda")
            sign = torch.randint(0, 2, (end,), generator=g, device="cuda", dtype=torch.uint8)
            s["m"] |= (sign * 128).mul_(s["m"] > 0)
        s["decay"] = torch.zeros(end, device="cuda")
        for x in _views(s["decay"], shapes, at)[:c["tables"]]:  # (vectors do not decay)
            x.fill_(DECAY)
        s["params"], s["grads"] = _views(s["p"], shapes, at), _views(s["grad"], shapes, at)
    if own:
        from paper_1410_8043_gb300 import esspt

        if c["kind"] in ("lookup", "embed_grad"):
            s["op"] = esspt.Embedding(c["T"], c["V"], c["D"], dtype=dtype, backward=c["kind"] == "embed_grad")
        elif c["kind"] == "norm":
            s["op"] = esspt.LayerNorm(c["T"], c["D"], dtype=dtype, weight_dtype=wtype, eps=NORM_EPS, backward=c["train"])
        else:
            copies = _views(s["copy"], shapes, at) if c["copy"] else None
            decay = [DECAY] * c["tables"] + [0.0] * c["vectors"]
            s["op"] = esspt.AdamW(s["params"], copies=copies, betas=(B1, B2), eps=EPS, weight_decay=decay,
                                  state_bits=c["bits"], seed=SEED)
            if c["bits"] == 32:
                s["op"].load(s["m"], s["v"], step=s["t"])
            else:
                s["op"].load(_held(s["m"], s["m_exp"], 3), _held(s["u"], s["u_exp"], 4), step=s["t"])
            for k in ("m", "v", "u", "m_exp", "u_exp", "decay"):
                s.pop(k, None)
    return s


# -- one pass -----------------------------------------------------------------
def _held(code, exp, bits):
    """The values that 8-bit codes stand for; `bits` of their fraction."""
    sign = (1 - (code & 128).float() / 64) if bits == 3 else 1.0
    code = (code & 127 if bits == 3 else code).int()
    x = ((code << (23 - bits)).view(-1, 128) + ((exp.int() - 15) << 23)[:, None]).view(torch.float32).view(-1)
    return torch.where(code > 0, x, 0.0) * sign


def _mix(x):
    x = ((x ^ (x >> 16)) * 0x5851F42D) & M32
    x = ((x ^ (x >> 15)) * 0x2545F491) & M32
    return x ^ (x >> 16)


def _hash(n, t):
    """32 bits for each of n values at step t."""
    k = _mix(torch.tensor([t & M32], device="cuda"))
    k = _mix((SEED & M32) ^ _mix((SEED >> 32) ^ k))
    i = torch.arange(n, device="cuda")
    return _mix((((i & M32) * 0x9E3779B1 + (i >> 32) * 0x85EBCA77) & M32) ^ k)


def _hold(x, bits, random):
    """8-bit codes of x >= 0 and its blocks' exponents; `random`: 16 bits for every value."""
    drop = 23 - bits
    b = x.view(torch.int32).view(-1, 128)
    exp = ((b.amax(dim=1) + ((1 << drop) - 1)) >> 23).clamp_(min=16)
    d = b - ((exp - 15) << 23)[:, None]
    least = (((exp - 15) << 23) + (1 << drop)).view(torch.float32)[:, None]
    random = random.view(-1, 128)
    code = (d + (random << (drop - 16))) >> drop
    if bits == 3:
        low = (x.view(-1, 128) >= (65536 - random).float() * (least / 65536)).int()
    else:
        low = (x.view(-1, 128) > 0).int()
    return torch.where(d < (1 << drop), low, code).view(-1).to(torch.uint8), exp.to(torch.uint8)


def _run_own(state):
    c, op = state["case"], state["op"]
    if c["kind"] == "lookup":
        return op.lookup(state["w"], state["ids"], scale=c["scale"])
    if c["kind"] == "embed_grad":
        return op.gradient(state["ids"], state["grad"], scale=c["scale"], grad_w=state.get("grad_w"), accumulate=c["add"])
    if c["kind"] == "norm":
        r = op.forward(state["x"], state["weight"], state["bias"])
        out = dict(y=r.y, mean=r.mean, rstd=r.rstd)
        if c["train"]:
            b = op.backward(state["dy"], state["x"], r.mean, r.rstd, state["weight"])
            out.update(grad_x=b.grad_x, grad_weight=b.grad_weight, grad_bias=b.grad_bias)
        return out
    op.step(state["grads"], LR)
    held = op.moments()
    return dict(p=state["p"], copy=state["copy"], m=held.m, second=held.second)


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    if c["kind"] == "lookup":
        ids = state["ids"].long()
        rows = state["w"][ids.clamp(min=0)].float().mul_(c["scale"])
        return torch.where((ids >= 0)[:, None], rows, 0.0).to(state["w"].dtype)
    if c["kind"] == "embed_grad":
        ids, grad = state["ids"].long(), state["grad"]
        rows = torch.where((ids >= 0)[:, None], grad.float(), 0.0).mul_(c["scale"])
        if c["add"]:
            total = state["grad_w"].float()
        else:
            total = torch.zeros((c["V"], c["D"]), device=grad.device)
        total.index_add_(0, ids.clamp(min=0), rows)
        return state["grad_w"].copy_(total) if c["add"] else total.to(grad.dtype)
    if c["kind"] == "norm":
        x, w = state["x"].float(), state["weight"].float()
        mean = x.mean(dim=1, keepdim=True)
        x = x - mean
        rstd = (x.square().mean(dim=1, keepdim=True) + NORM_EPS).rsqrt()
        x = x * rstd
        dtype, wtype = state["x"].dtype, state["weight"].dtype
        out = dict(y=(x * w + state["bias"].float()).to(dtype), mean=mean[:, 0], rstd=rstd[:, 0])
        if c["train"]:
            dy = state["dy"].float()
            g = dy * w
            dx = (g - g.mean(dim=1, keepdim=True) - x * (g * x).mean(dim=1, keepdim=True)) * rstd
            out.update(grad_x=dx.to(dtype), grad_weight=(dy * x).sum(dim=0).to(wtype), grad_bias=dy.sum(dim=0).to(wtype))
        return out
    state["t"] += 1
    p, g, t = state["p"], state["grad"].float(), state["t"]
    eight = c["bits"] == 8
    if eight:
        m, v = _held(state["m"], state["m_exp"], 3), _held(state["u"], state["u_exp"], 4).square_()
    else:
        m, v = state["m"], state["v"]
    m.mul_(B1).add_(g * (1 - B1))
    v.mul_(B2).add_((g * g).mul_(1 - B2))
    u = v.sqrt()
    step = (LR / (1 - B1**t) * m).div_((u / math.sqrt(1 - B2**t)).add_(EPS))
    p.mul_(1 - LR * state["decay"]).sub_(step)
    if eight:
        h = _hash(p.numel(), t)
        code, state["m_exp"] = _hold(m.abs(), 3, (h >> 16).int())
        state["m"] = torch.where((m < 0) & (code > 0), code | 128, code)
        state["u"], state["u_exp"] = _hold(u, 4, (h & 0xFFFF).int())
        m = _held(state["m"], state["m_exp"], 3).to(torch.bfloat16)  # (all of a code's bits)
        v = _held(state["u"], state["u_exp"], 4).to(torch.bfloat16)
    if c["copy"]:
        state["copy"].copy_(p)
    return dict(p=p, copy=state["copy"], m=m, second=v)


def work(case):
    c = case
    if c["kind"] == "adamw":
        n = sum(math.prod(s) for s in _layout(c)[0])
        grad, copy = (2, 2) if c["copy"] else (4, 0)
        # 8 bits: codes read and written, and the moments given out as 16-bit values
        return {"bytes": n * (8 + grad + copy + (16 if c["bits"] == 32 else 2 + 2 + 4)), "flops": 16 * n}
    size = 4 if c["dtype"] == "f32" else 2
    T, D = c["T"], c["D"]
    if c["kind"] == "norm":
        passes = 5 if c["train"] else 2  # x, y; x, dy, dx (a backward pass comes long after its forward pass)
        wsize = 4 if c["wtype"] == "f32" else 2
        return {"bytes": size * T * D * passes + 8 * T * (passes // 2) + 2 * wsize * D * (passes // 2),
                "flops": T * D * (24 if c["train"] else 8)}
    kept = T * (1.0 - c["pad"])
    # of ids with shares 1/k, the expected number of different ones
    u, V = 0.0, c["V"]
    edges = sorted({int(round(math.exp(math.log(V + 1) * i / 200))) for i in range(201)})
    for lo, hi in zip(edges, edges[1:]):
        share = math.log(hi / lo) / math.log(V + 1) / (hi - lo)
        u += (hi - lo) * -math.expm1(-kept * share)
    if c["kind"] == "lookup":
        return {"bytes": size * D * (u + T) + 4 * T, "flops": kept * D}
    return {"bytes": size * D * (kept + (2 * u if c["add"] else V)) + 4 * T, "flops": kept * D}


# -- in 64 bits ---------------------------------------------------------------
def _held64(code, exp, fraction):
    k = code.double()
    negative = k >= 128 if fraction == 8 else k < 0
    k = torch.where(negative, k - 128, k)
    e = torch.floor(k / fraction)
    x = (1 + (k - fraction * e) / fraction) * torch.exp2(e + exp.double().repeat_interleave(128) - 142)
    return torch.where(k > 0, torch.where(negative, -x, x), 0.0)


def _hold64(x, fraction, rho):
    """The values that x is held as, by arithmetic on values."""
    a = x.abs().view(-1, 128)
    low, e = torch.frexp(a.amax(dim=1, keepdim=True))
    e = torch.clamp(e - 1 + (2 * low > 2 - 1 / fraction).int(), min=-111)
    least = (1 + 1 / fraction) * torch.exp2(e.double() - 15)
    unit = torch.exp2(torch.frexp(a)[1].double() - 1) / fraction
    held = unit * torch.floor(a / unit + rho.view(-1, 128))
    below = least * (torch.floor(a / least + rho.view(-1, 128)) if fraction == 8 else (a > 0).double())
    return torch.where(a < least, below, held).view(-1) * torch.sign(x)


def exact(case, seed):
    c = case
    g = globals()
    before, g["own"] = own, False
    s = prepare(case, seed)
    g["own"] = before
    if c["kind"] == "lookup":
        out = torch.zeros((c["T"], c["D"]), dtype=torch.float64, device="cuda")
        at = (s["ids"] >= 0).nonzero()[:, 0]
        out[at] = c["scale"] * torch.index_select(s["w"], 0, s["ids"][at]).double()
        return out
    if c["kind"] == "embed_grad":
        at = (s["ids"] >= 0).nonzero()[:, 0]
        out = s["grad_w"].double() if c["add"] else torch.zeros((c["V"], c["D"]), dtype=torch.float64, device="cuda")
        return out.index_put_((s["ids"][at].long(),), c["scale"] * s["grad"][at].double(), accumulate=True)
    if c["kind"] == "norm":
        x, w, b = (s[k].double().requires_grad_(c["train"]) for k in ("x", "weight", "bias"))
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = 1 / torch.sqrt(var + NORM_EPS)
        y = torch.addcmul(b, (x - mean[:, None]) * rstd[:, None], w)
        out = dict(y=y.detach(), mean=mean.detach(), rstd=rstd.detach())
        if c["train"]:
            dx, dw, db = torch.autograd.grad((y * s["dy"].double()).sum(), (x, w, b))
            out.update(grad_x=dx, grad_weight=dw, grad_bias=db)
        return out
    t, grad = s["t"] + 1, s["grad"].double()
    if c["bits"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        m, v = _held64(s["m"], s["m_exp"], 8), _held64(s["u"], s["u_exp"], 16) ** 2
    m = torch.lerp(grad, m, B1)
    v = torch.lerp(grad * grad, v, B2)
    hat = (m / (1 - B1**t)) / ((v / (1 - B2**t)).sqrt() + EPS)
    p = s["p"].double()
    p = p - LR * (hat + s["decay"].double() * p)
    if c["bits"] == 8:
        h = _hash(p.numel(), t)
        rho = (h // 65536).double() / 65536, (h % 65536).double() / 65536
        m, v = _hold64(m, 8, rho[0]), _hold64(v.sqrt(), 16, rho[1])
    return dict(p=p, copy=p.clone() if c["copy"] else None, m=m, second=v)
