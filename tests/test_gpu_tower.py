"""The operators around a tower together, as the example calls them (-m gpu): embedding, norms and rotation, attention and its backward pass, the store,
clipping and orthogonalised steps."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from tower_ref import newton_schulz, rotate

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def trained():
    import boosted_histories as b
    import paper_1806_11248_amd as g
    ctx = g.Context(0)
    data = b.synthetic(1_500, seed=1)
    yield b, ctx, data, b.train(ctx, data, rounds=3, placed=True, orthogonal=True)
    ctx.close()


def test_it_runs(trained):
    b, ctx, data, (losses, trees, tower, tree_margin, tower_margin) = trained
    assert len(losses) == len(trees) == 3 and all(x == x and x < 10 for x in losses)
    assert bool(tower_margin.isfinite().all()) and all(bool(w.isfinite().all()) for w in tower.weights.values())


def test_the_towers_gradients_are_those_of_its_loss(trained):
    """Against automatic differentiation of the same tower in 64 bits, at the same rounded projection and the same rounded queries and keys behind their norms and
    turns.  What is left are roundings of 16-bit operands, some 2^-8 of a gradient each, of which there is one more than without norms; a twelfth of its
    length bounds them all, and no slip in passing gradients on is that small."""
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
    qkv = qkv + (torch.cat([*kept[7], kept[2]], dim=1).cpu().double() - qkv).detach()
    there, place = torch.ones(len(events), dtype=torch.bool), torch.arange(len(events)) - ptr[row_of]
    q, k, v = qkv.split([H, K, K], dim=1)
    q = rotate(q, w["q_norm"], tower.turns.cpu(), place, there, 1e-6, True)[0]
    k = rotate(k, w["k_norm"], tower.turns.cpu(), place, there, 1e-6, True)[0]
    for x, rounded in ((q, kept[0]), (k, kept[1])):
        assert float((x.detach() - rounded.cpu().double()).norm()) <= 2.0 ** -8 * float(x.detach().norm())
    edges = torch.tensor(tower.cuts)
    total = 0.0
    for r in range(len(ptr) - 1):
        n = int(ptr[r + 1] - ptr[r])
        margin64 = torch.zeros((), dtype=torch.float64)
        if n:
            rows = slice(int(ptr[r]), int(ptr[r + 1]))
            t = torch.arange(n)[None, :] - torch.arange(n)[:, None]
            heads = []
            for h in range(H):
                s = q[rows, h] @ k[rows, h // (H // K)].T * D ** -0.5 + w["bias"][:, h][torch.bucketize(t, edges, right=True)]
                heads.append(torch.softmax(s.masked_fill(t > 0, -float("inf")), 1) @ v[rows, h // (H // K)])
            margin64 = (torch.cat(heads, dim=1) @ w["head"]).mean()
        assert abs(float(margin64.detach()) - float(margin[r])) < 0.05 * (1 + abs(float(margin64.detach())))
        total = total + torch.nn.functional.softplus(margin64) - margin64 * float(y[r])
    total.backward()
    for n, t in w.items():
        assert float((tower.grads[n].cpu().double() - t.grad).norm()) <= float(t.grad.norm()) / 12, n


def test_the_projections_step_is_the_orthogonalised_moment(trained):
    b, ctx, _, (_, _, tower, *_) = trained
    data = b.synthetic(50, seed=4)
    X, ptr, events, row_of, y = (t.cuda() for t in data)
    before = tower.weights["project"].clone()
    margin, kept = tower.forward(ptr, row_of, events, int((ptr[1:] - ptr[:-1]).max()))
    tower.step(kept, (margin - y) / len(y), ptr, row_of, events, rate=0.5)
    want, bound = newton_schulz(tower.moments["project"][0].cpu(), 5, (3.4445, -4.7750, 2.0315))
    got = (before - tower.weights["project"]).cpu().double() / 0.5
    # the step's own error, and that of taking it from the weights and out again, in 32 bits
    assert float((got - want).norm()) <= bound + 4 * 2.0 ** -24 * float(before.norm()) / 0.5 + 2.0 ** -23 * float(want.norm())


def test_a_new_event_from_the_store_is_the_last_row_of_the_whole(trained):
    b, ctx, data, (_, _, tower, _, _) = trained
    X, ptr, events, row_of, y = (t.cuda() for t in data)
    rows = len(ptr) - 1
    new = torch.randint(0, 12, (rows,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    store = b.Store(tower, ptr, events, row_of)
    got = store.append(new)
    longer = torch.zeros_like(ptr)
    longer[1:] = ((ptr[1:] - ptr[:-1]) + 1).cumsum(0)
    all_events = torch.empty(int(longer[-1]), dtype=events.dtype, device="cuda")
    all_events[longer[row_of] + torch.arange(len(events), device="cuda") - ptr[row_of]] = events
    all_events[longer[1:] - 1] = new
    at = store.slots[:-1] + store.used - 1
    # what lies in the store is what the same projection gives at the same places, bit for bit
    (q, k, v), _ = tower.project(new)
    _, k = ctx.norm_rotate(q, k, *tower.norms(), positions=(store.used - 1).contiguous())
    assert torch.equal(store.k[at], k) and torch.equal(store.v[at], v)
    (q, k, v), x = tower.project(all_events)
    # and what whole histories have: products of 64 terms in 32 bits, which the library may add up in another order for another number of rows, and then
    # round to the neighbour, a step of 2^-7 at most
    last = longer[1:] - 1
    sums = 2 * 64 * 2.0 ** -24 * (x[last].abs() @ tower.weights["project"].abs()).view(len(last), -1, tower.head_dim)[:, -tower.kv_heads:]
    assert bool(((store.v[at].float() - v[last].float()).abs() <= 1.001 * (2.0 ** -7 * v[last].float().abs() + sums)).all())
    q, k = ctx.norm_rotate(q, k, *tower.norms(), q_ptr=longer)
    n = int((longer[1:] - longer[:-1]).max())
    whole = ctx.attention(q, k, v, **tower.args(q_ptr=longer, k_ptr=longer, max_q=n, max_k=n))[longer[1:] - 1]
    assert float((got.float() - whole.float()).abs().max()) <= 4 * 2.0 ** -8 * float(whole.float().abs().max())


def test_a_step_of_training_and_an_append_in_graphs():
    """Embedding, norms, attention, their backward passes, clipping and the orthogonalised step captured once and replayed with other events, between eager
    runs of the same, which use the context's workspaces."""
    import paper_1806_11248_amd as g
    side = torch.cuda.Stream()
    ctx = g.Context(0, stream=side)
    try:
        rng = torch.Generator().manual_seed(0)
        H, K, D, n_events = 4, 2, 32, 3_000
        table = torch.randn(40, 64, generator=rng).cuda()
        matrix = (torch.randn(64, (H + 2 * K) * D, generator=rng) / 8).cuda()
        ids = torch.randint(0, 40, (n_events,), generator=rng).cuda()
        ptr = torch.tensor([0, 1, 500, 1_700, n_events]).cuda()
        wq, wk, turns = torch.ones(D).cuda(), torch.ones(D).cuda(), g.rotation_turns(D)
        args = dict(q_ptr=ptr, k_ptr=ptr, max_q=1_300, max_k=1_300, causal=True)
        dout = torch.randn(n_events, H, D, generator=rng).to(torch.bfloat16).cuda()
        grads = [torch.zeros_like(table), torch.zeros_like(matrix)]
        step = torch.zeros_like(matrix)
        side.wait_stream(torch.cuda.current_stream())
        clip, ortho = ctx.gradient_list(grads), ctx.matrix_list([grads[1]], [step])

        def run():
            x = ctx.embedding(table, ids)
            raw_q, raw_k, v = (x @ matrix).to(torch.bfloat16).view(-1, H + 2 * K, D).split([H, K, K], dim=1)
            q, k = ctx.norm_rotate(raw_q, raw_k, wq, wk, turns, q_ptr=ptr)
            out, saved = ctx.attention(q, k, v, save=True, **args)
            dq, dk, dv, _ = ctx.attention_backward(dout, q, k, v, out, saved, **args)
            dq, dk, dwq, dwk = ctx.norm_rotate_backward(dq, dk, raw_q, raw_k, wq, wk, turns, q_ptr=ptr)
            dqkv = torch.cat([dq, dk, dv], dim=1).float().flatten(1)
            grads[1].copy_(x.t() @ dqkv)
            ctx.embedding_backward(dqkv @ matrix.t(), ids, out=grads[0])
            norm = ctx.clip_gradients(clip, 1.0)
            ctx.orthogonalise(ortho)
            return [out, dwq, dwk, norm, grads[0].clone(), step.clone()]

        with torch.cuda.stream(side):
            run()
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                captured = run()
            for seed in range(3):
                ids.copy_(torch.randint(0, 40, (n_events,), generator=torch.Generator().manual_seed(seed)))
                graph.replay()
                side.synchronize()
                got = [x.clone() for x in captured]
                eager = run()
                side.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(got, eager))
    finally:
        ctx.close()
