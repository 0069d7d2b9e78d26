"""The softmax operators over a catalogue: what a training or scoring program calls.

H [T, D] are rows that ask (user rows, hidden states), W [V, D] the rows of the
catalogue (item rows, a vocabulary), b the inverse temperature:

  s_tv = b h_t . w_v     lse_t = log sum_v exp s_tv     p_tv = exp(s_tv - lse_t)

  loss     softmax cross entropy: loss_t = lse_t - s_{t, y_t}.  A row whose
           target is negative is ignored: no loss, no gradient, whatever its h holds
  distill  from a teacher's top logits z_tk of the items id_tk (id < 0: no
           entry): q_t = softmax_k(b z_tk), loss_t = sum_k q_tk log(q_tk / p_t,id_tk).
           A row without entries is ignored

With `train` a pass returns the gradients of sum_t weight_t loss_t too:

  dh_t = b weight_t (sum_v p_tv w_v - sum_k q_tk w_id_tk)
  dw_v = b sum_t weight_t (p_tv - q_tv) h_t        (cross entropy: q_tv = [v = y_t])

The states hold rows as programs have them: some rows of a batch are padding
(their h was never written: NaN), popular items are targets far more often
than others, a teacher's lists are ragged.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _case(name, kind, T, V, D, dtype, train, top=1, ignored=0.1, stride=0, b=1.0):
    """T rows of width D against V items; top: entries of a teacher's list; ignored: share
    of padding rows; stride: values between the end of a row and the next one's start."""
    c = dict(kind=kind, T=T, V=V, D=D, dtype=dtype, train=train, top=top, ignored=ignored, stride=stride, b=b)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One user's choice scored against the mid catalogue (18k items, rank 100): latency.
        _case("loss_one_row", "loss", 1, 18_000, 100, "f32", False, ignored=0.0),
        # Eight users' choices against the largest catalogue (1M items, rank 64): one pass over W.
        _case("loss_few_rows_large", "loss", 8, 1_000_000, 64, "f32", False, ignored=0.0),
        # A step on the tiny workload's 1000 items, rank 16.
        _case("loss_train_tiny", "loss", 97, 1000, 16, "f32", True),
        # A step on the mid catalogue, rows in the table's fp32.
        _case("loss_train_mid", "loss", 4096, 18_000, 100, "f32", True),
        # A step on the largest catalogue, rank 64.
        _case("loss_train_large", "loss", 2048, 1_000_000, 64, "f32", True),
        # Half precision, as a network before the softmax hands rows over: odd sizes, rank 256,
        # half of the rows padding (prompts that are not learned from).
        _case("loss_train_bf16", "loss", 8195, 50_021, 256, "bf16", True, ignored=0.5),
        # The widest rows the table has, out of a wider buffer.
        _case("loss_train_wide_f16", "loss", 1021, 20_011, 512, "f16", True, stride=8),
        # Evaluation of a held-out set, forward alone.
        _case("loss_eval_bf16", "loss", 2003, 200_003, 128, "bf16", False),
        # Distillation on the tiny workload, short lists.
        _case("distill_tiny", "distill", 64, 1000, 16, "f32", True, top=8, b=0.5),
        # A step on the mid catalogue from lists of 32.
        _case("distill_mid", "distill", 4096, 18_000, 100, "f32", True, top=32, b=0.5),
        # Long lists over a large catalogue, half precision.
        _case("distill_large_bf16", "distill", 4001, 200_003, 64, "bf16", True, top=64, b=0.5),
        # Agreement with a teacher, forward alone.
        _case("distill_eval", "distill", 999, 100_003, 64, "f32", False, top=20, b=0.5),
    ]


def draw(rng):
    def logu(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["loss", "distill"])
    D = logu(8, 512)
    T, V = logu(1, 8192), logu(500, 1_000_000)
    while T * V * D > 130_000_000_000 or T * V > 2_000_000_000:
        T, V = max(1, T * 2 // 3), max(500, V * 2 // 3)
    return _case(None, kind, T, V, D, rng.choice(["f32", "f32", "bf16", "f16"]), rng.random() < 0.75,
                 top=logu(2, 100) if kind == "distill" else 1, ignored=rng.choice([0.0, 0.1, 0.5]),
                 stride=rng.choice([0, 0, 4, 3]), b=rng.choice([1.0, 0.5]))


# -- inputs -------------------------------------------------------------------
def _rows(g, n, D, stride, dtype, std):
    x = torch.randn((n, D + stride), generator=g, device="cuda", dtype=torch.float32).mul_(std).to(dtype)
    return x[:, :D]


def _items(g, shape, V):
    """Item ids, the k-th most popular with a share of about 1/k; ranks scattered over the ids."""
    rank = torch.rand(shape, generator=g, device="cuda", dtype=torch.float64).mul_(math.log(V)).exp_().long() - 1
    return torch.randperm(V, generator=g, device="cuda")[rank.clamp_(0, V - 1)].to(torch.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator("cuda")
    g.manual_seed(seed)
    dtype = TYPES[c["dtype"]]
    std = math.sqrt(2.0 / math.sqrt(c["D"]))  # logits of standard deviation 2
    h = _rows(g, c["T"], c["D"], c["stride"], dtype, std)
    w = _rows(g, c["V"], c["D"], c["stride"], dtype, std)
    weight = torch.rand(c["T"], generator=g, device="cuda") + 0.5
    pad = torch.rand(c["T"], generator=g, device="cuda") < c["ignored"]
    h[pad] = math.nan
    s = dict(case=c, h=h, w=w, weight=weight)
    if c["kind"] == "loss":
        s["targets"] = _items(g, (c["T"],), c["V"]).masked_fill_(pad, -1)
    else:
        ids = _items(g, (c["T"], c["top"]), c["V"]).sort(dim=1).values
        again = torch.zeros_like(ids, dtype=torch.bool)
        again[:, 1:] = ids[:, 1:] == ids[:, :-1]
        s["ids"] = ids.masked_fill_(again | pad[:, None], -1)
        s["logits"] = torch.randn((c["T"], c["top"]), generator=g, device="cuda").mul_(2.0).add_(6.0)
    if own:
        from paper_1410_8043_gb300 import esspt

        s["head"] = esspt.SoftmaxHead(c["T"], c["V"], c["D"], dtype=dtype, max_top=c["top"], backward=c["train"])
    return s


# -- one pass -----------------------------------------------------------------
def run(state):
    c = state["case"]
    if own:
        args = dict(weight=state["weight"], inv_temperature=c["b"], backward=c["train"])
        if c["kind"] == "loss":
            r = state["head"].loss(state["h"], state["w"], state["targets"], **args)
        else:
            r = state["head"].distill(state["h"], state["w"], state["ids"], state["logits"], **args)
        out = dict(loss=r.loss, lse=r.lse)
        if c["train"]:
            out.update(grad_h=r.grad_h, grad_w=r.grad_w)
        return out
    b, weight = c["b"], state["weight"]
    if c["kind"] == "loss":
        ids = state["targets"][:, None].long()
        present = ids >= 0
        q, log_q = present.float(), torch.zeros_like(ids, dtype=torch.float32)
        kept = present[:, 0]
    else:
        ids = state["ids"].long()
        z = torch.where(ids >= 0, state["logits"] * b, -math.inf)
        top = z.amax(dim=1, keepdim=True)
        kept = top[:, 0] > -math.inf
        z = z - torch.where(kept[:, None], top, 0.0)
        e = z.exp()
        total = torch.where(kept[:, None], e.sum(dim=1, keepdim=True), 1.0)
        q = e / total
        log_q = torch.where(q > 0, z - total.log(), 0.0)
    ids = ids.clamp(min=0)
    h = torch.where(kept[:, None], state["h"].float(), 0.0)
    w = state["w"].float()
    s = (h @ w.T).mul_(b)
    s_id = s.gather(1, ids)
    top = s.amax(dim=1, keepdim=True)
    p = s.sub_(top).exp_()
    total = p.sum(dim=1, keepdim=True)
    lse = (top + total.log())[:, 0]
    loss = torch.where(kept, (q * (log_q - s_id)).sum(dim=1) + lse, 0.0)
    out = dict(loss=loss, lse=torch.where(kept, lse, 0.0))
    if c["train"]:
        p.div_(total)
        rows = torch.arange(ids.shape[0], device=ids.device)[:, None].expand_as(ids)
        p.index_put_((rows, ids), -q, accumulate=True)
        p.mul_(torch.where(kept, weight * b, 0.0)[:, None])
        dtype = state["h"].dtype
        out.update(grad_h=(p @ w).to(dtype), grad_w=(p.T @ h).to(dtype))
    return out


def work(case):
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    T, V, D = c["T"] * (1.0 - c["ignored"]), c["V"], c["D"]
    passes = 2 if c["train"] else 1  # gradients are as large as what they belong to
    n = passes * size * D * (T + V) + 4 * c["T"] * (3 + (c["top"] if c["kind"] == "loss" else 2 * c["top"]))
    return {"bytes": n, "flops": (6 if c["train"] else 2) * T * V * D}


def exact(case, seed):
    """In fp64 by autograd from the definition, a few rows at a time."""
    c, s = case, prepare(case, seed)
    dev = s["h"].device
    if c["kind"] == "loss":
        ids, z = s["targets"][:, None].long(), torch.zeros((c["T"], 1), device=dev, dtype=torch.float64)
    else:
        ids, z = s["ids"].long(), s["logits"].double() * c["b"]
    loss = torch.zeros(c["T"], device=dev, dtype=torch.float64)
    lse = torch.zeros_like(loss)
    gh = torch.zeros((c["T"], c["D"]), device=dev, dtype=torch.float64)
    w = s["w"].double().requires_grad_(c["train"])
    gw = torch.zeros_like(w)
    live = ((ids >= 0) & (z > -math.inf)).any(dim=1).nonzero()[:, 0]
    for rows in live.split(max(1, 150_000_000 // c["V"])):
        h = s["h"][rows].double().requires_grad_(c["train"])
        log_q = torch.log_softmax(z[rows].masked_fill(ids[rows] < 0, -math.inf), dim=1)
        scores = c["b"] * torch.einsum("td,vd->tv", h, w)
        norm = torch.logsumexp(scores, dim=1)
        log_p = torch.gather(scores, 1, ids[rows].clamp(min=0)) - norm[:, None]
        part = torch.where(ids[rows] >= 0, log_q.exp() * (log_q.masked_fill(ids[rows] < 0, 0.0) - log_p), 0.0).sum(dim=1)
        loss[rows], lse[rows] = part.detach(), norm.detach()
        if c["train"]:
            dh, dw = torch.autograd.grad((part * s["weight"][rows].double()).sum(), (h, w))
            gh[rows] = dh
            gw += dw
    out = dict(loss=loss, lse=lse)
    if c["train"]:
        out.update(grad_h=gh, grad_w=gw.detach())
    return out
