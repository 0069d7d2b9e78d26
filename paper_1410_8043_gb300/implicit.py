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

The output is one JSON object per reported clock, one line each.
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
    args = ap.parse_args(argv)
    run(workload(args.workload), args.clocks, args.batch, args.eta, args.narrow, args.narrow_eta, args.top, args.every,
        lambda row: print(json.dumps(row), file=sys.stdout, flush=True))
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
