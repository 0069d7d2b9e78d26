"""Implicit feedback on the stale-synchronous table, and a narrow model learned from it.

The data are events "user i picked item j": the quarter of a workload's entries
with the highest values.  A model of rank K gives every user a softmax over all items by
the scores L_i . R_j, and each worker trains it as the paper's programs use a
parameter server (Sec. 4 "PS Interface"): in every clock it GETs the rows of a
batch of its users and of all items at its read version, takes the loss and its
gradients (`SoftmaxHead.loss`), INCs minus the step size times them, and CLOCKs.

A second, narrower model is then distilled (`SoftmaxHead.distill`) on a table of
its own from the first one's top scores for each user of a batch, as a service
would have stored them.

    python -m paper_1410_8043_gb300.implicit --workload tiny --clocks 40 --narrow 8

With `--dense` the same model is also trained by itself, without a table of versions:
rows are looked up (`Embedding`), normed (`LayerNorm`), scored against all items (`SoftmaxHead`), and the
gradients go back the same way to one `AdamW` step over all parameters (`DenseTrainer`).

    python -m paper_1410_8043_gb300.implicit --workload tiny --clocks 0 --narrow 0 --dense 40 --bits 8

The output is one JSON object per reported clock or step, one line each.
"""
from __future__ import annotations

import argparse
import contextlib
import json
import sys

import numpy as np
import torch

from . import esspt


class Trainer:
    """One model on a table: `n_users` + `n_items` rows of width K.

    Everything runs on the table's stream (`stream`, default: the current one at
    construction).  A call from another current stream comes after the work queued
    there, and that stream's later work after the call.
    """

    def __init__(self, n_users: int, n_items: int, K: int, P: int, s: int, batch: int, model: str = "ssp", seed: int = 1,
                 max_top: int = 1, init: float = 0.1, stream=None):
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self.n_users, self.P = n_users, P
        rng = np.random.default_rng(seed)
        with self._in_order():
            self.table = esspt.Table(n_users + n_items, K, P, s, model=model)
            self.head = esspt.SoftmaxHead(batch, n_items, K, max_top=max_top)
            self.table.table_init(rng.standard_normal((n_users + n_items, K), dtype=np.float32) * np.float32(init))
            self.items = torch.arange(n_users, n_users + n_items, dtype=torch.int32, device=self.table.device)

    @contextlib.contextmanager
    def _in_order(self):
        """On the table's stream, between what the current one has queued and what comes next."""
        current = torch.cuda.current_stream(self.stream.device)
        if current == self.stream:
            yield lambda x: x
            return
        self.stream.wait_stream(current)

        def hand_over(x):  # memory of one stream's, used by another
            x.record_stream(current)
            return x

        try:
            with torch.cuda.stream(self.stream):
                yield hand_over
        finally:
            current.wait_stream(self.stream)

    def _rows(self, worker: int, users):
        return self.table.get(worker, users)[0], self.table.get(worker, self.items)[0]

    def rows(self, worker: int, users):
        """The rows of `users` and of all items, at the worker's read version."""
        with self._in_order() as hand_over:
            return tuple(hand_over(x) for x in self._rows(worker, users))

    def _push(self, worker: int, users, r, eta: float):
        self.table.inc(worker, users, r.grad_h.mul_(-eta))
        self.table.inc(worker, self.items, r.grad_w.mul_(-eta))
        return r.loss

    def learn(self, worker: int, users, picks, eta: float):
        """One worker's part of a clock: steps of size eta down the sum of its batch's losses."""
        with self._in_order() as hand_over:
            h, w = self._rows(worker, users)
            return hand_over(self._push(worker, users, self.head.loss(h, w, picks), eta))

    def learn_from(self, worker: int, users, ids, logits, eta: float, inv_temperature: float = 1.0):
        """The same towards a teacher's top logits of the batch's users."""
        with self._in_order() as hand_over:
            h, w = self._rows(worker, users)
            return hand_over(self._push(worker, users, self.head.distill(h, w, ids, logits, inv_temperature=inv_temperature), eta))

    def close(self):
        self.head.poll()
        self.table.poll()
        self.head.close()
        self.table.close()


class DenseTrainer:
    """One model by itself: scores of all items from normed rows of a table of inputs.

    `n_inputs` rows (users, say) are the inputs, or, if it is None, the items themselves (what was picked
    before predicts what is picked next), whose rows then get both gradients.  Parameters are fp32; with a
    16-bit `dtype` the tables have copies of that type, on which everything but the norm's weights runs.  All handles run on
    the current stream at construction; a step with `lr` on the device may be captured in a CUDA graph.
    """

    def __init__(self, n_inputs: int | None, n_items: int, K: int, batch: int, dtype=torch.float32, state_bits: int = 32,
                 scale: float = 1.0, seed: int = 1, init: float = 0.1, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.0):
        self.tied, self.scale = n_inputs is None, scale
        g = torch.Generator("cuda").manual_seed(seed)
        rows = [n_items] if self.tied else [n_items, n_inputs]
        tables = [torch.randn((n, K), generator=g, device="cuda") * init for n in rows]
        self.weight, self.bias = torch.ones(K, device="cuda"), torch.zeros(K, device="cuda")
        self.params = tables + [self.weight, self.bias]
        run_on = tables if dtype is torch.float32 else [t.to(dtype) for t in tables]
        self.items, self.inputs = run_on[0], run_on[-1]
        copies = [None] * 4 if dtype is torch.float32 else run_on + [None, None]
        self.embedding = esspt.Embedding(batch, rows[-1], K, dtype=dtype)
        self.norm = esspt.LayerNorm(batch, K, dtype=dtype, weight_dtype=torch.float32)
        self.head = esspt.SoftmaxHead(batch, n_items, K, dtype=dtype)
        self.adamw = esspt.AdamW(self.params, copies=copies[:len(self.params)], betas=betas, eps=eps,
                                 weight_decay=[weight_decay] * len(tables) + [0.0, 0.0], state_bits=state_bits, seed=seed)

    def gradients(self, inputs, picks, weight=None):
        """Of the sum of a batch's (weighted) losses: the losses, and a gradient for each of `params`."""
        x = self.embedding.lookup(self.inputs, inputs, scale=self.scale)
        n = self.norm.forward(x, self.weight, self.bias)
        r = self.head.loss(n.y, self.items, picks, weight=weight)
        b = self.norm.backward(r.grad_h, x, n.mean, n.rstd, self.weight)
        if self.tied:
            tables = [self.embedding.gradient(inputs, b.grad_x, scale=self.scale, grad_w=r.grad_w, accumulate=True)]
        else:
            tables = [r.grad_w, self.embedding.gradient(inputs, b.grad_x, scale=self.scale)]
        return r.loss, tables + [b.grad_weight, b.grad_bias]

    def learn(self, inputs, picks, lr, weight=None):
        """One step on a batch of inputs (ids, negative ones padding) and the items picked after them."""
        loss, grads = self.gradients(inputs, picks, weight)
        self.adamw.step(grads, lr)
        return loss

    def close(self):
        self.embedding.poll()
        self.head.poll()
        for handle in (self.embedding, self.norm, self.head, self.adamw):
            handle.close()


def top_scores(h, r, top: int, piece: int = 65536):
    """The `top` largest scores h r^T of every row and their items (int32), by pieces of `r`,
    so that the scores of a large catalogue are never there as a whole."""
    values = h.new_empty((h.shape[0], 0))
    items = torch.empty((h.shape[0], 0), dtype=torch.int32, device=h.device)
    for begin in range(0, r.shape[0], piece):
        s = h @ r[begin:begin + piece].T
        best = torch.topk(s, min(top, s.shape[1]), dim=1)
        values, at = torch.topk(torch.cat([values, best.values], 1), min(top, values.shape[1] + best.values.shape[1]), dim=1)
        items = torch.cat([items, best.indices.int() + begin], 1).gather(1, at)
    return items, values


def batches(i, j, worker, P: int, batch: int, clocks: int, seed: int):
    """Per clock and worker a batch of the events of the worker's users (device int32)."""
    rng = np.random.default_rng(seed)
    mine = [np.flatnonzero(np.asarray(worker)[np.asarray(i)] == p) for p in range(P)]
    for _ in range(clocks):
        yield [(p, torch.as_tensor(i[k], dtype=torch.int32, device="cuda"),
                torch.as_tensor(j[k], dtype=torch.int32, device="cuda"))
               for p in range(P) if mine[p].size for k in [rng.choice(mine[p], batch)]]


def run(w, clocks: int, batch: int, eta: float, narrow: int, narrow_eta: float, top: int, every: int, emit) -> None:
    d = w.make_data()
    worker, _ = w.partition()
    M = w.n_items
    liked = np.flatnonzero(d.D >= np.quantile(d.D, 0.75))
    i, j = d.i[liked], d.j[liked]
    wide = Trainer(w.n_users, M, w.K, w.P, w.s, batch, model=w.model)
    for c, parts in enumerate(batches(i, j, worker, w.P, batch, clocks, 1), 1):
        losses = [wide.learn(p, u, k, eta) for p, u, k in parts]
        wide.table.clock()
        if c % every == 0 or c in (1, clocks):
            emit({"model": f"K={w.K}", "clock": c, "loss": float(torch.cat(losses).mean())})
    if narrow:
        small = Trainer(w.n_users, M, narrow, w.P, w.s, batch, model=w.model, seed=2, max_top=top)
        for c, parts in enumerate(batches(i, j, worker, w.P, batch, clocks, 2), 1):
            losses = []
            for p, u, _ in parts:
                h, r = wide.rows(p, u)
                losses.append(small.learn_from(p, u, *top_scores(h, r, top), narrow_eta))  # (what a service stores of the wide model)
            small.table.clock()
            if c % every == 0 or c in (1, clocks):
                emit({"model": f"K={narrow} from K={w.K}", "clock": c, "divergence": float(torch.cat(losses).mean())})
        small.close()
    wide.close()


def run_dense(w, steps: int, batch: int, lr: float, bits: int, dtype, every: int, emit) -> None:
    """The model by itself on the same events, all workers' batches together."""
    d = w.make_data()
    worker, _ = w.partition()
    liked = np.flatnonzero(d.D >= np.quantile(d.D, 0.75))
    model = DenseTrainer(w.n_users, w.n_items, w.K, batch * w.P, dtype=dtype, state_bits=bits)
    for c, parts in enumerate(batches(d.i[liked], d.j[liked], worker, w.P, batch, steps, 3), 1):
        loss = model.learn(torch.cat([u for _, u, _ in parts]), torch.cat([k for _, _, k in parts]), lr)
        if c % every == 0 or c in (1, steps):
            emit({"model": f"dense K={w.K}", "step": c, "loss": float(loss.mean())})
    model.close()


def main(argv=None) -> int:
    from gen import workload

    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--workload", default="tiny")
    ap.add_argument("--clocks", type=int, default=40)
    ap.add_argument("--batch", type=int, default=512, help="events per worker and clock")
    ap.add_argument("--eta", type=float, default=0.2, help="step size per event")
    ap.add_argument("--narrow", type=int, default=8, help="width of the distilled model (0: none)")
    ap.add_argument("--narrow-eta", type=float, default=0.05,
                    help="its step size per event (a popular item is on most lists: its row's steps add up)")
    ap.add_argument("--top", type=int, default=20, help="length of the teacher's lists")
    ap.add_argument("--every", type=int, default=10, help="clocks between reports")
    ap.add_argument("--dense", type=int, default=0, help="steps of the model by itself, by AdamW (0: none)")
    ap.add_argument("--lr", type=float, default=0.01, help="its step size")
    ap.add_argument("--bits", type=int, default=32, choices=(32, 8), help="bits of its moments")
    ap.add_argument("--dtype", default="float32", choices=("float32", "bfloat16", "float16"), help="what it runs in")
    args = ap.parse_args(argv)

    def emit(row):
        print(json.dumps(row), file=sys.stdout, flush=True)

    if args.clocks:
        run(workload(args.workload), args.clocks, args.batch, args.eta, args.narrow, args.narrow_eta, args.top, args.every, emit)
    if args.dense:
        run_dense(workload(args.workload), args.dense, args.batch, args.lr, args.bits, getattr(torch, args.dtype), args.every, emit)
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
