"""The example that trains trees and an attention tower on the same gradients (-m gpu)."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def trained():
    import boosted_histories as b
    import paper_1806_11248_amd as g
    ctx = g.Context(0)
    data = b.synthetic(4_000, seed=1)
    yield b, ctx, data, b.train(ctx, data, rounds=12)
    ctx.close()


def test_both_learn_more_than_the_trees_alone(trained):
    b, ctx, data, (losses, trees, tower, *_) = trained
    alone = b.train(ctx, data, rounds=12, with_tower=False)[0]
    assert losses[-1] < losses[0] and losses[-1] < alone[-1] - 0.03
    assert len(trees) == 12 and float(tower.weights["bias"].abs().max()) > 0.0


def test_the_towers_gradients_are_those_of_its_loss(trained):
    """Against automatic differentiation of the same tower in 64 bits, taken at the same rounded queries, keys and values.  What is left are
    roundings of 16-bit operands, some 2^-8 of a gradient each; a sixteenth of its length bounds them all, and no slip in passing gradients on
    is that small."""
    b, ctx, _, (_, _, tower, *_) = trained
    data = b.synthetic(60, seed=3)
    X, ptr, events, row_of, y = (t.cuda() for t in data)
    margin, kept = tower.forward(ptr, row_of, events, int((ptr[1:] - ptr[:-1]).max()))
    pairs = ctx.gradients("logistic", margin, y)
    tower.step(kept, pairs[:, 0].contiguous(), ptr, row_of, events, rate=0.0, max_norm=1e30)

    _, ptr, events, row_of, y = data
    w = {n: t.cpu().double().requires_grad_() for n, t in tower.weights.items()}
    H, K, D = tower.heads, tower.kv_heads, tower.head_dim
    qkv = (w["embed"][events] @ w["project"]).view(-1, H + 2 * K, D)
    rounded = torch.cat(kept[:3], dim=1).cpu().double()
    qkv = qkv + (rounded - qkv).detach()
    edges = torch.tensor(tower.cuts)
    total = 0.0
    for r in range(len(ptr) - 1):
        n = int(ptr[r + 1] - ptr[r])
        margin64 = torch.zeros((), dtype=torch.float64)
        if n:
            part = qkv[ptr[r]:ptr[r + 1]]
            t = torch.arange(n)[None, :] - torch.arange(n)[:, None]
            heads = []
            for h in range(H):
                s = part[:, h] @ part[:, H + h // (H // K)].T * D ** -0.5 + w["bias"][:, h][torch.bucketize(t, edges, right=True)]
                heads.append(torch.softmax(s.masked_fill(t > 0, -float("inf")), 1) @ part[:, H + K + h // (H // K)])
            margin64 = (torch.cat(heads, dim=1) @ w["head"]).mean()
        assert abs(float(margin64) - float(margin[r])) < 0.05 * (1 + abs(float(margin64)))
        total = total + torch.nn.functional.softplus(margin64) - margin64 * float(y[r])
    total.backward()
    for n, t in w.items():
        assert float((tower.grads[n].cpu().double() - t.grad).norm()) <= float(t.grad.norm()) / 16, n


def test_a_new_event_from_the_store_is_the_last_row_of_the_whole(trained):
    b, ctx, data, (_, _, tower, _, _) = trained
    X, ptr, events, row_of, y = (t.cuda() for t in data)
    rows = len(ptr) - 1
    new = torch.randint(0, 12, (rows,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    got = b.Store(tower, ptr, events, row_of).append(new)
    longer = torch.zeros_like(ptr)
    longer[1:] = ((ptr[1:] - ptr[:-1]) + 1).cumsum(0)
    all_events = torch.empty(int(longer[-1]), dtype=events.dtype, device="cuda")
    all_events[longer[row_of] + torch.arange(len(events), device="cuda") - ptr[row_of]] = events
    all_events[longer[1:] - 1] = new
    (q, k, v), _ = tower.project(all_events)
    n = int((longer[1:] - longer[:-1]).max())
    whole = ctx.attention(q, k, v, **tower.args(q_ptr=longer, k_ptr=longer, max_q=n, max_k=n))[longer[1:] - 1]
    # each side rounds its probabilities and its result once: twice the largest value's half unit in the last place, and as much for the sums
    assert float((got.float() - whole.float()).abs().max()) <= 4 * 2.0 ** -8 * float(whole.float().abs().max())
