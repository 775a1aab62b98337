"""A user's history beside the samples' bags: a small sequence tower trained and served with the library's calls on histories, its output
the dense features of the per-task meta step.

  train   history tokens -> rows (inputs | gates) -> recurrence -> candidates' queries attend to its states -> score against the
          candidate's target row -> binary cross-entropy; gradients back through every call, tables updated in place
  serve   one more event a user: its row, one step of the recurrence, the state appended to the user's slot of a cache; a candidate's query
          over the slots
  meta    the tower's vector of a user as the dense features of that user's samples in GMeta.meta_step (which returns no gradient with respect to
          them: the tower is trained on its own objective)

    python examples/history_tower.py [--steps 30] [--users 256] [--items 20000]
"""
from __future__ import annotations

import argparse
import os
import sys
from types import SimpleNamespace

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2401_04338_amd import GMeta  # noqa: E402

HEADS, KV_HEADS, HEAD_DIM = 4, 2, 32
CHANNELS, WIDTH = KV_HEADS * HEAD_DIM, HEADS * HEAD_DIM     # of the recurrence's states, of a query
EMB_SCALE = 4.0


class HistoryTower:
    """Two tables: an event's row is (input | gate) of the recurrence, a candidate's (query | target)."""

    def __init__(self, gm: GMeta, items: int, gen: torch.Generator):
        self.gm, self.items = gm, items
        self.events = torch.randn(items, 2 * CHANNELS, device="cuda", generator=gen) * 0.1
        self.events[:, CHANNELS:] += 2.0 / EMB_SCALE        # (gates begin open: a memory of some eight events)
        self.candidates = torch.randn(items, 2 * WIDTH, device="cuda", generator=gen) * 0.1

    def encode(self, tokens, offsets, longest):
        rows = self.gm.seq_embed(self.events, tokens, EMB_SCALE, dtype=torch.bfloat16)
        x, gate = rows[:, :CHANNELS], rows[:, CHANNELS:]
        h, last = self.gm.seq_scan(x, gate, offsets, longest)
        return x, gate, h, last

    def look(self, candidates, h, q_offsets, k_offsets, longest_q, longest_k, k_lengths=None):
        rows = self.gm.seq_embed(self.candidates, candidates, EMB_SCALE, dtype=torch.bfloat16)
        q, target = rows[:, :WIDTH].unflatten(1, (HEADS, HEAD_DIM)), rows[:, WIDTH:]
        kv = h.view(-1, KV_HEADS, HEAD_DIM)
        o, lse = self.gm.seq_attend(q, kv, kv, q_offsets, k_offsets, longest_q, longest_k, k_lengths=k_lengths)
        return q, target, kv, o, lse

    def train_step(self, batch, lr: float) -> torch.Tensor:
        b, gm = batch, self.gm
        x, gate, h, _ = self.encode(b.tokens, b.offsets, b.longest)
        q, target, kv, o, lse = self.look(b.candidates, h, b.q_offsets, b.offsets, b.longest_q, b.longest)
        flat = o.reshape(-1, WIDTH)
        logit = (flat.float() * target.float()).sum(1)
        loss = torch.nn.functional.binary_cross_entropy_with_logits(logit, b.labels)
        d = ((torch.sigmoid(logit) - b.labels) / len(logit))[:, None]
        # the gradient of a table's rows lies as the rows do: halves of one array
        d_cand, d_event = torch.empty(len(q), 2 * WIDTH, dtype=torch.bfloat16, device="cuda"), torch.empty(len(x), 2 * CHANNELS, dtype=torch.bfloat16, device="cuda")
        d_cand[:, WIDTH:] = d * flat.float()
        dout = (d * target.float()).to(torch.bfloat16).view_as(o)
        dk, dv = torch.empty_like(kv), torch.empty_like(kv)
        gm.seq_attend_grad(dout, q, kv, kv, o, lse, b.q_offsets, b.offsets, b.longest_q, b.longest,
                           out=(d_cand[:, :WIDTH].unflatten(1, (HEADS, HEAD_DIM)), dk, dv))
        gm.seq_scan_grad((dk + dv).view(-1, CHANNELS), x, gate, h, b.offsets, b.longest, out=(d_event[:, :CHANNELS], d_event[:, CHANNELS:]))
        gm.seq_embed_grad(d_cand, b.candidates, self.items, -lr * EMB_SCALE, table=self.candidates)
        gm.seq_embed_grad(d_event, b.tokens, self.items, -lr * EMB_SCALE, table=self.events)
        return loss


class Server:
    """Users' states and a slot of `room` encoded events each."""

    def __init__(self, tower: HistoryTower, users: int, room: int):
        self.tower, self.users, self.room = tower, users, room
        self.state = torch.zeros(users, CHANNELS, device="cuda")
        self.cache = torch.zeros(users, room, CHANNELS, dtype=torch.bfloat16, device="cuda")
        self.lengths = torch.zeros(users, dtype=torch.int64, device="cuda")
        self.slots = torch.arange(users + 1, device="cuda") * room
        self.ones = torch.arange(users + 1, device="cuda")

    def event(self, tokens):
        """One event of every user (-1: none): the state and the cache of the others go on."""
        gm, came = self.tower.gm, tokens >= 0
        rows = gm.seq_embed(self.tower.events, tokens, EMB_SCALE, dtype=torch.bfloat16)
        state = self.state.clone()
        h = gm.seq_scan_step(rows[:, :CHANNELS], rows[:, CHANNELS:], state)
        self.state = torch.where(came[:, None], state, self.state)
        users = torch.arange(self.users, device="cuda")
        at = self.lengths.clamp(max=self.room - 1)
        self.cache[users, at] = torch.where(came[:, None], h, self.cache[users, at])
        self.lengths = torch.where(came, (self.lengths + 1).clamp(max=self.room), self.lengths)

    def vectors(self, candidates):
        """What the tower makes of one candidate a user."""
        return self.tower.look(candidates, self.cache, self.ones, self.slots, 1, self.room, k_lengths=self.lengths)[3].reshape(self.users, WIDTH)


def make_batch(users: int, items: int, gen, rng, longest: int = 96, candidates: int = 8):
    """Histories of 0 .. longest events of a taste (a block of items) each; half of the candidates are of the user's taste."""
    lens = rng.integers(0, longest + 1, size=users)
    lens[0] = 0
    off, n, m = np.concatenate([[0], np.cumsum(lens)]), int(lens.sum()), users * candidates
    block = max(1, items // 16)
    taste = torch.from_numpy(rng.integers(0, 16, size=users)).cuda()
    own = lambda who, k: taste[who] * block + torch.randint(0, block, (k,), device="cuda", generator=gen)  # noqa: E731
    who, cand = torch.from_numpy(np.repeat(np.arange(users), lens)).cuda(), torch.arange(users, device="cuda").repeat_interleave(candidates)
    tokens = own(who, n).to(torch.int32)
    tokens[torch.rand(n, device="cuda", generator=gen) < 0.02] = -1           # events whose item is not known any more
    labels = (torch.arange(m, device="cuda") % 2).float()
    other = torch.randint(0, items, (m,), device="cuda", generator=gen)
    return SimpleNamespace(tokens=tokens, offsets=torch.from_numpy(off).cuda(), longest=longest, candidates=torch.where(labels > 0, own(cand, m), other).to(torch.int32),
                           q_offsets=torch.arange(users + 1, device="cuda") * candidates, longest_q=candidates, labels=labels, lens=lens)


def meta_step_with(vectors: torch.Tensor, gen, tasks: int = 4):
    """The users' vectors as dense features of the meta step: `tasks` tasks of support and query samples."""
    per = len(vectors) // (2 * tasks)
    fields, rows, dim = 2, 50, 8
    dims = [fields * dim + WIDTH, 32, 1]
    gm = GMeta(fields, [rows] * fields, dim, WIDTH, dims, workspace_bytes=64 << 20)

    def samples(v):
        n = len(v)
        return SimpleNamespace(task_offsets=np.arange(tasks + 1, dtype=np.int64) * per, bag_offsets=torch.arange(n * fields + 1, device="cuda"),
                               indices=torch.randint(0, rows, (n * fields,), device="cuda", generator=gen).to(torch.int32),
                               dense=v.float().contiguous(), labels=(torch.rand(n, device="cuda", generator=gen) < 0.3).float())
    params = SimpleNamespace(emb=torch.randn(fields * rows, dim, device="cuda", generator=gen) * 0.05,
                             W=[torch.randn(a, b, device="cuda", generator=gen) / a ** 0.5 for a, b in zip(dims[:-1], dims[1:])],
                             b=[torch.zeros(b, device="cuda") for b in dims[1:]])
    out = gm.meta_step(samples(vectors[:tasks * per]), samples(vectors[tasks * per:2 * tasks * per]), params, 0.01, 1, 2)
    gm.close()
    return float(out["loss"])


def run(steps: int = 30, users: int = 256, items: int = 20_000, lr: float = 20.0, seed: int = 0, say=print):
    """Returns (losses, largest difference between served and trained vectors relative to the largest vector entry, meta loss)."""
    gen, rng = torch.Generator(device="cuda").manual_seed(seed), np.random.default_rng(seed)
    gm = GMeta(1, [16], 4, 0, [4, 1], workspace_bytes=256 << 20)
    gm.configure("wait", 0)
    tower, losses = HistoryTower(gm, items, gen), []
    batch = make_batch(users, items, gen, rng)
    for i in range(steps):
        losses.append(tower.train_step(batch, lr))
        if i % 10 == 9:
            gm.wait()
            say(f"step {i + 1}: loss {float(losses[-1]):.4f}")
    gm.wait()
    losses = [float(x) for x in losses]
    # serve the same histories event by event
    server = Server(tower, users, batch.longest)
    for t in range(int(batch.lens.max())):
        at = batch.offsets[:-1] + t
        here = torch.from_numpy(batch.lens > t).cuda()
        server.event(torch.where(here, batch.tokens[at.clamp(max=len(batch.tokens) - 1)], -1))
    first = batch.candidates.view(users, -1)[:, 0].contiguous()
    served = server.vectors(first)
    # (an unknown item has no row in the cache: the trained tower sees it as a row of zeros, so compare the users without one)
    _, _, h, _ = tower.encode(batch.tokens, batch.offsets, batch.longest)
    trained = tower.look(first, h, server.ones, batch.offsets, 1, batch.longest)[3].reshape(users, WIDTH)
    gm.wait()
    unknown = torch.zeros(users, device="cuda").index_add_(0, torch.from_numpy(np.repeat(np.arange(users), batch.lens)).cuda(), (batch.tokens < 0).float())
    known = unknown == 0
    off = float((served.float() - trained.float())[known].abs().max() / trained.float().abs().max())
    say(f"served against trained vectors of {int(known.sum())} users: off by {off:.2e}")
    meta = meta_step_with(served, gen)
    say(f"meta step on the users' vectors: loss {meta:.4f}")
    gm.close()
    return losses, off, meta


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--users", type=int, default=256)
    ap.add_argument("--items", type=int, default=20_000)
    a = ap.parse_args()
    run(a.steps, a.users, a.items)
