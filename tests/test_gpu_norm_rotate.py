"""Head norms with rotation, the way into the store, and the backward pass, against plain 64-bit forms (-m gpu).  Bounds: tower_ref."""
import math

import pytest
import torch

from tower_ref import TINY, U, places, rotate, rotate_gradient

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    import paper_1806_11248_amd as g
    c = g.Context(0)
    yield c
    c.close()


def _inputs(rows, heads, kv_heads, dim, dtype, seed=0, fused=True):
    rng = torch.Generator().manual_seed(seed)
    size = torch.exp(torch.randn(heads + 2 * kv_heads, 1, generator=rng))
    x = (torch.randn(rows, heads + 2 * kv_heads, dim, generator=rng) * size).to(dtype).cuda()
    q, k, v = x.split([heads, kv_heads, kv_heads], dim=1)
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    return q, k, v, 1 + 0.3 * torch.randn(dim, generator=rng).cuda(), 1 + 0.3 * torch.randn(dim, generator=rng).cuda()


def _turns(turned):
    import paper_1806_11248_amd as g
    return g.rotation_turns(turned)


def _close(got, want, bound):
    err = (got.cpu().double() - want).abs()
    tol = 1.001 * (U[got.dtype] * want.abs() + (1 + U[got.dtype]) * bound) + TINY[got.dtype]
    assert bool((err <= tol).all()), (float((err - tol).max()), int((err > tol).sum()))


def _check(ctx, q, k, v, wq, wk, turns, there, position, eps=1e-6, halves=True, backward=True, **args):
    dim = q.shape[2]
    host = [torch.ones(dim) if w is None else w.cpu() for w in (wq, wk)]
    t = torch.zeros(0, dtype=torch.float64) if turns is None else turns.cpu()
    q_out, k_out, v_out = ctx.norm_rotate(q, k, wq, wk, turns, v=v, eps=eps, halves=halves, **args)
    for got, x, w in ((q_out, q, host[0]), (k_out, k, host[1])):
        _close(got, *rotate(x.cpu(), w, t, position, there, eps, halves))
    assert torch.equal(v_out.cpu(), torch.where(there[:, None, None], v.cpu(), torch.zeros((), dtype=v.dtype)))
    pair = ctx.norm_rotate(q, k, wq, wk, turns, eps=eps, halves=halves, **args)
    assert torch.equal(pair[0], q_out) and torch.equal(pair[1], k_out)
    if backward:
        rng = torch.Generator().manual_seed(77)
        dq_out, dk_out = (torch.randn(x.shape, generator=rng).to(x.dtype).cuda() for x in (q, k))
        got = ctx.norm_rotate_backward(dq_out, dk_out, q, k, wq, wk, turns, eps=eps, halves=halves, **args)
        for dx, dw, x, w, d in ((got[0], got[2], q, host[0], dq_out), (got[1], got[3], k, host[1], dk_out)):
            want, bound, of_weight, of_bound = rotate_gradient(d.cpu(), x.cpu(), w, t, position, there, eps, halves)
            _close(dx, want, bound)
            _close(dw, of_weight, of_bound)
    return q_out, k_out


@pytest.mark.parametrize("rows,heads,kv_heads,dim,turned", [
    (1, 1, 1, 8, 8), (1, 8, 2, 64, 64), (5, 6, 2, 80, 32), (7, 3, 3, 40, 40), (64, 5, 5, 24, 8), (33, 16, 4, 128, 128), (129, 2, 1, 96, 48), (50, 40, 8, 16, 16),
    (20, 1, 1, 120, 0), (300, 32, 8, 128, 120), (9, 70, 1, 8, 8), (2, 7, 5, 56, 56), (1000, 4, 2, 32, 32)])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("halves", [True, False])
def test_packed(ctx, rows, heads, kv_heads, dim, turned, dtype, halves):
    q, k, v, wq, wk = _inputs(rows, heads, kv_heads, dim, dtype, rows, fused=rows % 2 == 0)
    position = torch.arange(rows)
    _check(ctx, q, k, v, wq, wk, _turns(turned), torch.ones(rows, dtype=torch.bool), position, halves=halves)


def test_without_weights_or_turns(ctx):
    q, k, v, wq, wk = _inputs(50, 4, 2, 64, BF16)
    there, position = torch.ones(50, dtype=torch.bool), torch.arange(50)
    _check(ctx, q, k, v, None, wk, _turns(64), there, position)
    _check(ctx, q, k, v, wq, None, None, there, position)
    _check(ctx, q, k, v, None, None, None, there, position, eps=0.5)


@pytest.mark.parametrize("wide", [False, True])
def test_far_positions(ctx, wide):
    """Explicit ones, negative and up to where 32 bits have no fraction of a revolution left."""
    rng = torch.Generator().manual_seed(5)
    position = torch.cat([torch.randint(-(1 << 31), 1 << 31, (60,), generator=rng), torch.tensor([0, 1, -1, (1 << 31) - 1, -(1 << 31)])])
    q, k, v, wq, wk = _inputs(65, 4, 2, 64, F16)
    device = position.cuda() if wide else position.int().cuda()
    _check(ctx, q, k, v, wq, wk, _turns(64), torch.ones(65, dtype=torch.bool), position, positions=device)


@pytest.mark.parametrize("lengths,before,behind", [([3], 0, 0), ([5, 0, 1, 7, 0], 0, 0), ([0, 0], 2, 3), ([2, 9, 4], 3, 5), ([1] * 200, 0, 1), ([0] * 70 + [4, 40], 1, 0),
                                                   ([11] * 5000, 0, 7)])
def test_sequences(ctx, lengths, before, behind):
    """Ragged rows; those of no sequence, before the first and behind the last, get zeros, also where they hold NaN."""
    ptr = [before]
    for n in lengths:
        ptr.append(ptr[-1] + n)
    rows = ptr[-1] + behind
    for heads, kv_heads, dim, eps in ((4, 2, 64, 1e-6), (1, 1, 16, 0.0), (3, 1, 40, 0.0)) if rows < 10_000 else ((1, 1, 8, 1e-6),):
        q, k, v, wq, wk = _inputs(rows, heads, kv_heads, dim, BF16, rows)
        there, position, _ = places(rows, ptr)
        for x in (q, k, v):
            x[~there.cuda()] = math.nan
        clean = [x.cpu().nan_to_num(0.0) for x in (q, k, v)]
        q_out, k_out, v_out = ctx.norm_rotate(q, k, wq, wk, _turns(dim), v=v, eps=eps, q_ptr=torch.tensor(ptr).cuda())
        for got, x, w in ((q_out, clean[0], wq), (k_out, clean[1], wk)):
            _close(got, *rotate(x, w.cpu(), _turns(dim).cpu(), position, there, eps, True))
        assert torch.equal(v_out.cpu(), clean[2])
        d = torch.full_like(q, math.nan), torch.full_like(k, math.nan)
        for x in d:
            x[there.cuda()] = 1.0
        dq, dk, dwq, dwk = ctx.norm_rotate_backward(*d, q, k, wq, wk, _turns(dim), eps=eps, q_ptr=torch.tensor(ptr).cuda())
        for got, dw, x, w in ((dq, dwq, clean[0], wq), (dk, dwk, clean[1], wk)):
            want, bound, of_weight, of_bound = rotate_gradient(torch.ones(x.shape), x, w.cpu(), _turns(dim).cpu(), position, there, eps, True)
            _close(got, want, bound)
            _close(dw, of_weight, of_bound)


@pytest.mark.parametrize("new,used,room", [([1, 1, 1], [4, 1, 9], [5, 3, 9]), ([3, 0, 6, 1], [3, 2, 10, 1], [4, 2, 30, 8]), ([4, 2], [2, 2], [8, 8]),
                                           ([2, 2], [9, 2], [4, 4]), ([1] * 100, [7] * 100, [9] * 100)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_store(ctx, new, used, room, dtype):
    """Keys and values go to the last places in use of their slot, with more new rows than places in use, and more in use than the slot has, among them; all
    other rows of the stores stay."""
    ptr, slots = [0], [2]
    for n, r in zip(new, room):
        ptr.append(ptr[-1] + n)
        slots.append(slots[-1] + r)
    rows, store_rows = ptr[-1], slots[-1] + 3
    for heads, kv_heads, dim in ((8, 2, 64), (2, 2, 80), (1, 1, 8)):
        q, k, v, wq, wk = _inputs(rows, heads, kv_heads, dim, dtype, rows)
        ks, vs = (torch.randn(store_rows, kv_heads, dim, generator=torch.Generator().manual_seed(i)).to(dtype).cuda() for i in (1, 2))
        before = ks.cpu(), vs.cpu()
        there, position, to = places(rows, ptr, slots, used)
        args = dict(k_ptr=torch.tensor(slots).cuda(), k_len=torch.tensor(used, dtype=torch.int32).cuda())
        if len(set(new)) > 1:
            args["q_ptr"] = torch.tensor(ptr).cuda()
        q_out, k_out, v_out = ctx.norm_rotate(q, k, wq, wk, _turns(dim), v=v, k_out=ks, v_out=vs, **args)
        assert k_out is ks and v_out is vs
        _close(q_out, *rotate(q.cpu(), wq.cpu(), _turns(dim).cpu(), position, there, 1e-6, True))
        kept = torch.ones(store_rows, dtype=torch.bool)
        kept[to[to >= 0]] = False
        assert torch.equal(ks.cpu()[kept], before[0][kept]) and torch.equal(vs.cpu()[kept], before[1][kept])
        want, bound = rotate(k.cpu(), wk.cpu(), _turns(dim).cpu(), position, there, 1e-6, True)
        _close(ks[to[to >= 0].cuda()], want[to >= 0], bound[to >= 0])
        assert torch.equal(vs.cpu()[to[to >= 0]], v.cpu()[to >= 0])
        # the same positions without a store
        packed = ctx.norm_rotate(q, k, wq, wk, _turns(dim), **args)
        assert torch.equal(packed[0], q_out) and torch.equal(packed[1][(to >= 0).cuda()], ks[to[to >= 0].cuda()])


def test_store_without_pointers(ctx):
    """Slots of one length; only keys; and positions of their own."""
    q, k, v, wq, wk = _inputs(6, 4, 2, 32, BF16)
    ks = torch.zeros(3 * 7, 2, 32, dtype=BF16, device="cuda")
    used = [5, 2, 7]
    there, position, to = places(6, None, None, used, 3, 21)
    q_out, _ = ctx.norm_rotate(q, k, wq, wk, _turns(32), k_len=torch.tensor(used, dtype=torch.int32).cuda(), k_out=ks)
    want, bound = rotate(k.cpu(), wk.cpu(), _turns(32).cpu(), position, there, 1e-6, True)
    _close(ks[to.cuda()], want, bound)
    own = torch.tensor([100, 3, 9, 4, 1 << 20, 0])
    ctx.norm_rotate(q, k, wq, wk, _turns(32), k_len=torch.tensor(used, dtype=torch.int32).cuda(), k_out=ks, positions=own.int().cuda())
    want, bound = rotate(k.cpu(), wk.cpu(), _turns(32).cpu(), own, there, 1e-6, True)
    _close(ks[to.cuda()], want, bound)


def test_store_pointers_that_lie_outside(ctx):
    """Slots beyond the store, negative ones and negative lengths hold no rows: nothing is written there, or anywhere."""
    q, k, v, wq, wk = _inputs(4, 2, 1, 16, BF16)
    for slots, used in (([0, 5, 100, 105, 1 << 40], [5, 50, 5, 5]), ([-4, 0, -9, 5, 10], [4, 1, 3, -3]), ([9, 4, 4, 20, 20], [1, 1, 1, 1]),
                        ([3, -(1 << 63) + 1, 5, -(1 << 63), 4], [2, 2, 2, 2])):
        ks, vs = torch.full((12, 1, 16), 3.0, dtype=BF16, device="cuda"), torch.full((12, 1, 16), 3.0, dtype=BF16, device="cuda")
        ctx.norm_rotate(q, k, wq, wk, _turns(16), v=v, k_ptr=torch.tensor(slots).cuda(), k_len=torch.tensor(used, dtype=torch.int32).cuda(), k_out=ks, v_out=vs)
        written = (vs != 3.0).flatten(1).any(1)
        for s in range(4):
            lo, n = slots[s], min(slots[s + 1] - slots[s], used[s])
            if n > 0 and lo >= 0 and lo + n <= 12:
                assert torch.equal(vs[lo + n - 1], v[s])
                written[lo + n - 1] = False
        assert not bool(written.any())
        # and without lengths, where the differences of the last ones pass 64 bits
        ks.fill_(3.0)
        ctx.norm_rotate(q, k, wq, wk, _turns(16), k_ptr=torch.tensor(slots).cuda(), k_out=ks)
        for s in range(4):
            if 0 <= slots[s] < slots[s + 1] <= 12:
                ks[slots[s + 1] - 1] = 3.0
        assert bool((ks == 3.0).all())


def test_in_place_and_parts_of_one_tensor(ctx):
    q, k, v, wq, wk = _inputs(77, 8, 2, 64, BF16)
    want = ctx.norm_rotate(q, k, wq, wk, _turns(64))
    rng = torch.Generator().manual_seed(1)
    d = [torch.randn(x.shape, generator=rng).to(BF16).cuda() for x in (q, k)]
    grads = ctx.norm_rotate_backward(*d, q, k, wq, wk, _turns(64))
    whole = torch.zeros(77, 12, 64, dtype=BF16, device="cuda")
    parts = whole.split([8, 2, 2], dim=1)
    again = ctx.norm_rotate_backward(*d, q, k, wq, wk, _turns(64), dq=parts[0], dk=parts[1])
    assert again[0] is parts[0] and all(torch.equal(a, b) for a, b in zip(again, grads)) and bool((parts[2] == 0).all())
    same = ctx.norm_rotate_backward(*[x.clone() for x in d], q, k, wq, wk, _turns(64))
    assert all(torch.equal(a, b) for a, b in zip(same, grads))
    e = [x.clone() for x in d]
    ctx.norm_rotate_backward(*e, q, k, wq, wk, _turns(64), dq=e[0], dk=e[1])
    assert torch.equal(e[0], grads[0]) and torch.equal(e[1], grads[1])
    ctx.norm_rotate(q, k, wq, wk, _turns(64), q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_rows_of_extreme_size(ctx):
    """Zeros, the smallest and the largest numbers of the types, and what is not finite, which stays in its head."""
    for dtype in (BF16, F16):
        q = torch.ones(8, 2, 32, dtype=dtype, device="cuda")
        k = q.clone()
        q[0] = 0
        q[1] = torch.finfo(dtype).tiny
        q[2] = 1e18 if dtype is BF16 else 6e4
        q[3, 0, 5] = math.nan
        q[4, 1, 5] = math.inf
        there = torch.ones(8, dtype=torch.bool)
        q_out, _ = ctx.norm_rotate(q, k, None, None, _turns(32))
        want, bound = rotate(q.cpu(), torch.ones(32), _turns(32).cpu(), torch.arange(8), there, 1e-6, True)
        fine = torch.tensor([0, 1, 2, 5, 6, 7])
        _close(q_out[fine.cuda()], want[fine], bound[fine])
        assert bool(q_out[3, 0].isnan().any()) and bool(q_out[3, 1].isfinite().all()) and bool(q_out[4, 0].isfinite().all())
        assert not bool(q_out[4, 1].isfinite().all())
        d = torch.ones_like(q)
        dq, dk, dwq, _ = ctx.norm_rotate_backward(d, d, q[fine.cuda()].repeat(2, 1, 1)[:8], k, None, None, _turns(32))
        assert bool(dq.isfinite().all()) and bool(dwq.isfinite().all())


def test_a_gradient_against_differences(ctx):
    """Of a 64-bit form that the results were compared with, at steps along single elements and weights."""
    rng = torch.Generator().manual_seed(3)
    x = torch.randn(3, 2, 16, generator=rng, dtype=torch.float64)
    d = torch.randn(3, 2, 16, generator=rng, dtype=torch.float64)
    w = 1 + 0.2 * torch.randn(16, generator=rng, dtype=torch.float64)
    t, there, position = _turns(16).cpu(), torch.ones(3, dtype=torch.bool), torch.tensor([0, 5, 1000])
    for halves in (True, False):
        def loss(x, w):
            return float((rotate(x, w, t, position, there, 1e-3, halves)[0] * d).sum())
        dx, _, dw, _ = rotate_gradient(d, x, w, t, position, there, 1e-3, halves)
        for at in ((0, 0, 0), (1, 1, 7), (2, 0, 15)):
            step = torch.zeros_like(x)
            step[at] = 1e-5
            assert abs((loss(x + step, w) - loss(x - step, w)) / 2e-5 - float(dx[at])) < 1e-6
        for e in (0, 9):
            step = torch.zeros_like(w)
            step[e] = 1e-5
            assert abs((loss(x, w + step) - loss(x, w - step)) / 2e-5 - float(dw[e])) < 1e-6


@pytest.mark.parametrize("rows", [40, 20_000])
def test_the_same_on_every_run_and_in_graphs(rows):
    import paper_1806_11248_amd as g
    side = torch.cuda.Stream()
    own = g.Context(0, stream=side)
    try:
        q, k, v, wq, wk = _inputs(rows, 8, 2, 64, BF16)
        turns = _turns(64)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            def both():
                out = own.norm_rotate(q, k, wq, wk, turns)
                return (*out, *own.norm_rotate_backward(*out, q, k, wq, wk, turns))
            both()
            side.synchronize()
            graphs = []
            for _ in range(2):
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    got = both()
                graphs.append((graph, got))
            for step in range(3):
                q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(step)))
                for graph, _ in graphs:
                    graph.replay()
                eager = both()
                side.synchronize()
                for _, got in graphs:
                    assert all(torch.equal(a, b) for a, b in zip(got, eager))
    finally:
        own.close()


def test_refusals(ctx):
    import paper_1806_11248_amd as g
    q, k, v, wq, wk = _inputs(6, 4, 2, 64, BF16)
    t = _turns(64)
    ptr, used = torch.tensor([0, 2, 6]).cuda(), torch.tensor([2, 4], dtype=torch.int32).cuda()
    store = torch.zeros(10, 2, 64, dtype=BF16, device="cuda")
    for args, kw in (((q.cpu(), k, wq, wk, t), {}), ((q[0], k, wq, wk, t), {}), ((q, k[:5], wq, wk, t), {}), ((q, k.half(), wq, wk, t), {}),
                     ((q, k, wq[:32], wk, t), {}), ((q, k, wq, wk.double(), t), {}), ((q, k, wq, wk, t.float()), {}), ((q, k, wq, wk, t.cpu()), {}),
                     ((q, k, wq, wk, t), dict(q_ptr=ptr.int())), ((q, k, wq, wk, t), dict(q_ptr=ptr, k_len=used[:1])),
                     ((q, k, wq, wk, t), dict(k_len=used.repeat(2))), ((q, k, wq, wk, t), dict(positions=torch.zeros(5, dtype=torch.int32).cuda())),
                     ((q, k, wq, wk, t), dict(positions=torch.zeros(6).cuda())), ((q, k, wq, wk, t), dict(v_out=store, k_out=store, k_len=used, q_ptr=ptr)),
                     ((q, k, wq, wk, t), dict(k_out=store)), ((q, k, wq, wk, t), dict(k_out=store[:, :1], k_len=used, q_ptr=ptr)),
                     ((q, k, wq, wk, t), dict(k_out=store[:9], k_len=used, q_ptr=ptr)), ((q, k, wq, wk, t), dict(q_out=q.half())),
                     ((q.transpose(1, 2), k, wq, wk, t), {})):
        with pytest.raises(TypeError):
            ctx.norm_rotate(*args, **kw)
    for args, kw, code in (((q.float(), k.float(), wq, wk, t), {}, "EUNSUPPORTED"), ((q, k, wq, wk, t), dict(eps=-1.0), "EINVAL"), ((q, k, wq, wk, t), dict(eps=math.nan), "EINVAL"),
                           ((q, k, wq, wk, _turns(72)), {}, "EINVAL"), ((q, k, wq, wk, _turns(12)), {}, "EUNSUPPORTED"),
                           ((q[..., :60], k[..., :60], None, None, _turns(8)), {}, "EUNSUPPORTED"),
                           ((q, k, wq, wk, t), dict(q_out=q[:1].expand(6, 4, 64)), "EINVAL")):
        with pytest.raises(g.GbtError) as e:
            ctx.norm_rotate(*args, **kw)
        assert e.value.code == getattr(g.binding, code)
    with pytest.raises(TypeError):
        ctx.norm_rotate_backward(q, k[:3], q, k, wq, wk, t)


def test_what_attention_reads(ctx):
    """A run as serving makes it: whole histories into the store, then one new event each, against the whole histories at once."""
    rng = torch.Generator().manual_seed(9)
    lengths = [5, 1, 30, 64]
    H, K, D = 4, 2, 32
    turns, wq, wk = _turns(D), 1 + 0.1 * torch.randn(D, generator=rng).cuda(), 1 + 0.1 * torch.randn(D, generator=rng).cuda()
    ptr = torch.tensor([0] + torch.tensor(lengths).cumsum(0).tolist())
    x = torch.randn(int(ptr[-1]), H + 2 * K, D, generator=rng).to(BF16).cuda()
    q, k, v = x.split([H, K, K], dim=1)
    whole_q, whole_k = ctx.norm_rotate(q, k, wq, wk, turns, q_ptr=ptr.cuda())
    want = ctx.attention(whole_q, whole_k, v, q_ptr=ptr.cuda(), k_ptr=ptr.cuda(), max_q=64, max_k=64, causal=True)
    slots = torch.tensor([0] + (torch.tensor(lengths) + 3).cumsum(0).tolist()).cuda()
    ks, vs = (torch.full((int(slots[-1]), K, D), math.nan, dtype=BF16, device="cuda") for _ in range(2))
    # all but the last event of each, then the last
    first = torch.cat([torch.arange(int(a), int(b) - 1) for a, b in zip(ptr[:-1], ptr[1:])]).cuda()
    before = torch.tensor([0] + (torch.tensor(lengths) - 1).cumsum(0).tolist()).cuda()
    used = torch.tensor([n - 1 for n in lengths], dtype=torch.int32).cuda()
    ctx.norm_rotate(q[first], k[first], wq, wk, turns, v=v[first], q_ptr=before, k_ptr=slots, k_len=used, k_out=ks, v_out=vs)
    last = (ptr[1:] - 1).cuda()
    used += 1
    new_q, _, _ = ctx.norm_rotate(q[last], k[last], wq, wk, turns, v=v[last], k_ptr=slots, k_len=used, k_out=ks, v_out=vs)
    assert torch.equal(new_q, whole_q[last])
    got = ctx.attention(new_q, ks, vs, q_ptr=torch.arange(5).cuda(), k_ptr=slots, k_len=used, max_q=1, max_k=67, causal=True)
    # probabilities of few rows are operands in two parts, those of blocks in one: a rounding of half a step each, and out's
    assert bool(((got.float() - want[last].float()).abs() <= 3 * U[BF16] * v.float().abs().max()).all())
