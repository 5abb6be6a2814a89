"""Boosted trees over a table whose rows come with a history of events, and a small attention tower over the histories.

Both learn the same thing from the same gradients: a row's margin is what the trees make of its columns plus what the tower makes of its
events, and every round takes the gradient pairs of that margin, grows one tree on them, and takes a few steps with the tower.

  whole histories   Context.attention over ragged rows, a learned bias for each bucket of distance; its gradients from
                    Context.attention_backward, scaled down together by Context.clip_gradients
  a new event       appended to a store with room, and read by one query row a history

    python examples/boosted_histories.py            # on an MI355X; prints the loss of trees alone, and of both
"""
from __future__ import annotations

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1806_11248_amd as g   # noqa: E402


def synthetic(rows, seed=0, columns=8, kinds=12, longest=90):
    """Columns, ragged histories of event kinds, and labels that depend on both: on two columns, and on how lately events of one kind came
    before events of another."""
    rng = torch.Generator().manual_seed(seed)
    X = torch.randn(rows, columns, generator=rng)
    lengths = torch.randint(0, longest + 1, (rows,), generator=rng)
    ptr = torch.zeros(rows + 1, dtype=torch.int64)
    ptr[1:] = lengths.cumsum(0)
    events = torch.randint(0, kinds, (int(ptr[-1]),), generator=rng)
    row_of = torch.repeat_interleave(torch.arange(rows), lengths)
    since = torch.full((rows,), longest, dtype=torch.int64)
    place = torch.arange(len(events)) - ptr[row_of]
    hit = events == 3
    since.scatter_reduce_(0, row_of[hit], (lengths[row_of] - 1 - place)[hit], "amin")     # events since the last of kind 3
    logit = 1.5 * X[:, 0] * X[:, 1] + 2.0 * (since < 4).float() - 1.0 * (since > 15).float() - 0.3
    y = (torch.rand(rows, generator=rng) < torch.sigmoid(logit)).float()
    return X, ptr, events, row_of, y


class Tower:
    """Embedded events, one projection to queries, keys and values, attention, and a weight for each element of each head's mean."""

    def __init__(self, ctx, kinds, width=64, heads=4, kv_heads=2, head_dim=32, buckets=24, far=64, seed=0):
        rng = torch.Generator(device="cuda").manual_seed(seed)
        self.ctx, self.heads, self.kv_heads, self.head_dim = ctx, heads, kv_heads, head_dim
        self.cuts = g.distance_cuts(buckets, far)
        out = (heads + 2 * kv_heads) * head_dim

        def normal(*shape, scale):
            return torch.randn(*shape, generator=rng, device="cuda") * scale

        self.weights = dict(embed=normal(kinds, width, scale=1.0), project=normal(width, out, scale=width ** -0.5),
                            bias=torch.zeros(buckets, heads, device="cuda"), head=normal(heads * head_dim, scale=(heads * head_dim) ** -0.5))
        self.grads = {n: torch.zeros_like(w) for n, w in self.weights.items()}
        self.plan = ctx.gradient_list(self.grads.values())
        self.moments = {n: (torch.zeros_like(w), torch.zeros_like(w)) for n, w in self.weights.items()}
        self.steps = 0

    def project(self, events):
        """(q, k, v) as parts of one tensor, and the embedded events."""
        w = self.weights
        x = w["embed"][events]
        qkv = (x @ w["project"]).to(torch.bfloat16).view(-1, self.heads + 2 * self.kv_heads, self.head_dim)
        return qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1), x

    def args(self, **rows):
        return dict(rows, causal=True, bias=self.weights["bias"], cuts=self.cuts)

    def margins(self, out, ptr, row_of, rows):
        """The mean over a history's events of what the head makes of them; 0 for a history without events."""
        score = out.float().flatten(1) @ self.weights["head"]
        count = (ptr[1:] - ptr[:-1]).clamp_min(1).float()
        return torch.zeros(rows, device="cuda").index_add_(0, row_of, score) / count

    def forward(self, ptr, row_of, events, longest):
        (q, k, v), x = self.project(events)
        args = self.args(q_ptr=ptr, k_ptr=ptr, max_q=longest, max_k=longest)
        out, saved = self.ctx.attention(q, k, v, save=True, **args)
        margin = self.margins(out, ptr, row_of, len(ptr) - 1)
        return margin, (q, k, v, x, out, saved, args)

    def step(self, kept, dmargin, ptr, row_of, events, rate=0.01, max_norm=1.0):
        """One step of Adam on the clipped gradients, from the gradient of each row's margin.  Returns the global norm (on the device)."""
        q, k, v, x, out, saved, args = kept
        w, d = self.weights, self.grads
        count = (ptr[1:] - ptr[:-1]).clamp_min(1).float()
        each = (dmargin / count)[row_of]                                                   # of each event's score
        d["head"].copy_(each @ out.float().flatten(1))
        dout = (each[:, None] * w["head"]).to(torch.bfloat16).view_as(out)
        dq, dk, dv, dbias = self.ctx.attention_backward(dout, q, k, v, out, saved, **args)
        dqkv = torch.cat([dq, dk, dv], dim=1).float().flatten(1)
        d["bias"].copy_(dbias)
        d["project"].copy_(x.t() @ dqkv)
        d["embed"].zero_().index_add_(0, events, dqkv @ w["project"].t())
        norm = self.ctx.clip_gradients(self.plan, max_norm)
        self.steps += 1
        for n, grad in d.items():
            m, s = self.moments[n]
            m.lerp_(grad, 0.1)
            s.lerp_(grad * grad, 0.01)
            w[n] -= rate * (m / (1 - 0.9 ** self.steps)) / ((s / (1 - 0.99 ** self.steps)).sqrt() + 1e-8)
        return norm


class Store:
    """Keys and values of every history's events, with room for more, and each history's sum of event scores."""

    def __init__(self, tower, ptr, events, row_of, room=16):
        self.tower = tower
        lengths = ptr[1:] - ptr[:-1]
        self.slots = torch.zeros_like(ptr)
        self.slots[1:] = (lengths + room).cumsum(0)
        self.used = lengths.to(torch.int32)
        total = int(self.slots[-1])
        self.longest = int(lengths.max()) + room
        shape = (total, tower.kv_heads, tower.head_dim)
        self.k, self.v = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        (q, k, v), _ = tower.project(events)
        at = self.slots[row_of] + torch.arange(len(events), device="cuda") - ptr[row_of]
        self.k[at], self.v[at] = k, v

    def append(self, events):
        """One new event for every history, (their last free place must not be taken); its attention output."""
        t = self.tower
        (q, k, v), _ = t.project(events)
        at = self.slots[:-1] + self.used
        self.k[at], self.v[at] = k, v
        self.used += 1
        ptr = torch.arange(len(events) + 1, device="cuda")
        return t.ctx.attention(q, self.k, self.v, **t.args(q_ptr=ptr, k_ptr=self.slots, k_len=self.used, max_q=1, max_k=self.longest))


def loss(margin, y):
    return float(torch.nn.functional.binary_cross_entropy_with_logits(margin, y))


def train(ctx, data, rounds=20, tower_steps=4, eta=0.3, depth=4, bins=64, with_tower=True):
    """Rounds of one tree and a few steps of the tower.  Returns (loss of each round, trees, tower, quantised matrix's parts, margins)."""
    X, ptr, events, row_of, y = (t.cuda() for t in data)
    rows, columns = X.shape
    longest = int((ptr[1:] - ptr[:-1]).max())
    cuts, nb, packed, bits, _, missing = ctx.quantise_packed(X.contiguous(), max_bins=bins)
    params = g.make_params(max_depth=depth, max_bins=bins, eta=eta, objective="logistic")
    tower = Tower(ctx, int(events.max()) + 1) if with_tower else None
    trees, losses = [], []
    tree_margin, tower_margin = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    for _ in range(rounds):
        if with_tower:
            for _ in range(tower_steps):
                tower_margin, kept = tower.forward(ptr, row_of, events, longest)
                pairs = ctx.gradients("logistic", tree_margin + tower_margin, y)
                tower.step(kept, pairs[:, 0] / rows, ptr, row_of, events)
            tower_margin, _ = tower.forward(ptr, row_of, events, longest)
        pairs = ctx.gradients("logistic", tree_margin + tower_margin, y)
        tree, _, _ = ctx.grow_tree(packed, bits, rows, columns, missing, nb, cuts, pairs, params, want_leaf=False, want_rows=False)
        ctx.predict([tree], tree_margin, eta, packed=packed, bits=bits, missing_sym=missing, n=rows, F=columns)
        trees.append(tree)
        losses.append(loss(tree_margin + tower_margin, y))
    return losses, trees, tower, tree_margin, tower_margin


def main(rows=20_000):
    ctx = g.Context(0)
    data = synthetic(rows)
    alone = train(ctx, data, with_tower=False)[0]
    both, _, tower, _, _ = train(ctx, data)
    print(f"{rows} rows, {len(data[2])} events; logistic loss after 20 rounds: trees alone {alone[-1]:.4f}, with the tower {both[-1]:.4f}")
    X, ptr, events, row_of, y = (t.cuda() for t in data)
    store = Store(tower, ptr, events, row_of)
    out = store.append(torch.full((rows,), 3, device="cuda"))
    score = out.float().flatten(1) @ tower.weights["head"]
    print(f"a new event of kind 3 scores {float(score.mean()):+.3f} on average, read against {int(store.used.sum())} stored events")
    assert math.isfinite(float(score.sum()))


if __name__ == "__main__":
    main()
