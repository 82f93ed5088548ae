"""A small training step that uses a table and the sequence tower together, as a model over user histories would.

The events of every history are looked up unpooled (bags of one) in an embedding table; a gated recurrence runs over each
history; causal attention with a learned relative position bias reads the states; the last position scores the next event.  The table
is updated by row-wise Adagrad on the touched rows, the dense parameters by AdamW with 8-bit moments.

With --items the last position scores a catalogue instead: its state and what attention read are added and normalised, and the log probability of the item
that came next is the loss, with the best items of a larger tower (here: made up) as a second one.  recommend() serves the best items, the norm in 8 bits.

    python examples/history_tower.py [--steps 30] [--items 5000]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2305_01515_b200 import binding as mb  # noqa: E402
from paper_2305_01515_b200 import head as hd  # noqa: E402
from paper_2305_01515_b200 import sequence as sq  # noqa: E402
from paper_2305_01515_b200 import workload as wl  # noqa: E402
from paper_2305_01515_b200.harness import DeviceModel  # noqa: E402


class HistoryTower:
    """Histories of one length L, so that the attention needs no padding; the recurrence itself takes ragged ones."""

    def __init__(self, rows=20000, D=64, H=4, S=64, L=96, lr=3e-3, state_bits=8, seed=0, items=0):
        self.D, self.H, self.S, self.L = D, H, S, L
        tables = wl._finish_tables([wl.TableSpec(rows, D, 1, 0.9)], np.random.default_rng(seed))
        self.spec = wl.ModelSpec("history", tables, wl.FP32, S * L, "fixed", seed=seed)
        self.table = DeviceModel(self.spec)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.buckets = mb.RelposBuckets(sq.log_bucket_starts(16, 64), causal=True)
        shapes = dict(gates=(D, 2 * D), qkv=(D, 3 * D), bias=(self.buckets.rows, H), out=(D, D), shift=(D,))
        if items:                                                         # a norm of ones and the items' vectors in the place of a target's
            del shapes["out"], shapes["shift"]
            shapes.update(items=(D, items), norm=(D,))
        self.p = {k: (torch.randn(*s, generator=g, device="cuda") * (0.0 if k in ("bias", "shift") else s[0] ** -0.5)).requires_grad_()
                  for k, s in shapes.items()}
        if items:
            self.p["norm"].data.fill_(1.0)
        self.optimizer = sq.AdamW(list(self.p.values()), lr=lr, state_bits=state_bits)
        self.bag = torch.arange(S * L + 1, device="cuda")                 # bags of one event
        self.offsets = torch.arange(0, S * L + 1, L, device="cuda")       # histories

    def read(self, events):
        """events [S L, D] -> what the last position of each history reads of the others, and its own state, [S, D] each."""
        p, S, L, H, d = self.p, self.S, self.L, self.H, self.D // self.H
        gate, value = (events @ p["gates"]).chunk(2, dim=1)               # column ranges of one projection
        states, _ = sq.gated_recurrence(gate, value, self.offsets)
        q, k, v = (states @ p["qkv"]).view(S, L, 3, H, d).permute(2, 0, 3, 1, 4)
        scores = sq.add_relpos_bias(q @ k.transpose(2, 3) * d ** -0.5, p["bias"], self.buckets)
        read = (torch.softmax(scores, -1) @ v).transpose(1, 2).reshape(S, L, self.D)
        return read[:, -1], states.view(S, L, self.D)[:, -1]

    def forward(self, events):
        """What the last position of each history makes of it, [S, D]."""
        read, state = self.read(events)
        return (read + state) @ self.p["out"] + self.p["shift"]

    def scores(self, events):
        """Scores of the items of the catalogue for the next event of each history."""
        read, state = self.read(events)
        x, _ = hd.rms_norm(read, self.p["norm"], state)
        return x @ self.p["items"]

    def next_loss(self, events, item, teacher=None):
        """Loss [S] of the items that came next (negative: none did); teacher: (index, scores, rest) of a larger tower's best items."""
        scores = self.scores(events)
        loss = -hd.log_probs(scores, item).logp
        return loss if teacher is None else loss + hd.distill_loss(scores, teacher[0], teacher[1], teacher[2], scale=0.5)

    def next_step(self, indices, item, teacher=None):
        """One training step on the items that came next."""
        N = self.S * self.L
        events = self.table.forward(indices, self.bag, N).requires_grad_()
        loss = self.next_loss(events, item, teacher).mean()
        self.optimizer.zero_grad()
        loss.backward()
        self.optimizer.step()
        self.table.backward(indices, self.bag, N, events.grad, lr=0.02)
        return loss.detach()

    @torch.no_grad()
    def recommend(self, indices, k):
        """The k best next items of each history, and their log probabilities."""
        read, state = self.read(self.table.forward(indices, self.bag, self.S * self.L))
        codes, scales, _ = hd.rms_norm_8bit(read, self.p["norm"], state)
        best = hd.log_probs(hd.rows_from_8bit(codes, scales, dtype=torch.float32) @ self.p["items"], top_k=k)
        return best.top_index, best.top_logp

    def step(self, indices, target):
        """One training step; target [S, D]: what the next event looks like."""
        N = self.S * self.L
        events = self.table.forward(indices, self.bag, N).requires_grad_()
        loss = (self.forward(events) - target).square().mean()
        self.optimizer.zero_grad()
        loss.backward()
        self.optimizer.step()
        self.table.backward(indices, self.bag, N, events.grad, lr=0.02)
        return loss.detach()

    def close(self):
        self.table.close()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--items", type=int, default=0, help="score a catalogue of so many items")
    a = ap.parse_args()
    tower = HistoryTower(items=a.items)
    g = torch.Generator(device="cuda").manual_seed(1)
    indices = torch.randint(int(tower.spec.rows[0]), (tower.S * tower.L,), generator=g, device="cuda")
    target = torch.randn(tower.S, tower.D, generator=g, device="cuda")
    if a.items:
        item = torch.randint(a.items, (tower.S,), generator=g, device="cuda")
        best = torch.rand(tower.S, a.items, generator=g, device="cuda").topk(min(16, a.items))[1]
        teacher = best, torch.randn(best.shape, generator=g, device="cuda"), torch.zeros(tower.S, device="cuda")
    for k in range(a.steps):
        loss = tower.next_step(indices, item, teacher) if a.items else tower.step(indices, target)
        if k % 5 == 0 or k + 1 == a.steps:
            print(f"step {k:3d}  loss {float(loss):.4f}")
    if a.items:
        print("best next items of the first history:", tower.recommend(indices, min(5, a.items))[0][0].tolist())
    tower.close()


if __name__ == "__main__":
    main()
