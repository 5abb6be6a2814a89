"""Head norms with rotation: inputs of which a wave has many rows, and what only the C entry points can be asked for (-m gpu).  Bounds: tower_ref."""
import ctypes as C

import pytest
import torch

from tower_ref import TINY, TURN, U, places, rotate, rotate_gradient

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    import paper_1806_11248_amd as g
    c = g.Context(0)
    yield c
    c.close()


def _turns(turned):
    import paper_1806_11248_amd as g
    return g.rotation_turns(turned)


def _close(got, want, bound):
    got, want, bound = got.cpu().double(), want.cpu(), bound.cpu()
    u, tiny = U[BF16], TINY[BF16]
    err = (got - want).abs()
    assert bool((err <= 1.001 * (u * want.abs() + (1 + u) * bound) + tiny).all())


@pytest.mark.parametrize("n_seq,each,room", [(1, 7, 7), (3, 4, 6), (3, 6, 4), (5, 1, 1), (2, 300, 301)])
@pytest.mark.parametrize("ragged", [False, True])
def test_a_store_of_equal_slots_all_in_use(ctx, n_seq, each, room, ragged):
    """A store with neither k_ptr nor k_len: slots of out_rows / n_seq rows, and nk = nq: row i goes to row i of its slot, if that has one."""
    b = __import__("paper_1806_11248_amd").binding
    H, K, D = 4, 2, 32
    rows = n_seq * each
    rng = torch.Generator().manual_seed(rows)
    q, k, v = (torch.randn(rows, h, D, generator=rng).to(BF16).cuda() for h in (H, K, K))
    weight = (1 + 0.3 * torch.randn(D, generator=rng)).cuda()
    turns = _turns(D)
    ptr = [each * s for s in range(n_seq + 1)]
    if ragged and n_seq > 1:
        ptr[1] = min(each + 1, ptr[2])
    q_ptr = torch.tensor(ptr).cuda()
    ks, vs = (torch.full((n_seq * room, K, D), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    q_out = torch.empty_like(q)
    p = b.NormRotateParams(1, H, K, D, D, 1, 1, n_seq, 4, 1e-6, rows, n_seq * room, q_ptr.data_ptr() if ragged else None, None, None, None, weight.data_ptr(),
                           weight.data_ptr(), turns.data_ptr())
    heads = [b.Heads(t.data_ptr(), t.stride(0), t.stride(1)) for t in (q, k, v, q_out, ks, vs)]
    assert ctx.lib.gbt_norm_rotate(ctx.h, C.byref(p), *[C.byref(h) for h in heads]) == b.OK
    there, position, _ = places(rows, ptr)
    to = torch.full((rows,), -1)
    for s in range(n_seq):
        for i in range(min(room, ptr[s + 1] - ptr[s])):
            to[ptr[s] + i] = s * room + i
    _close(q_out, *rotate(q.cpu(), weight.cpu(), turns.cpu(), position, there, 1e-6, True))
    want, bound = rotate(k.cpu(), weight.cpu(), turns.cpu(), position, there, 1e-6, True)
    goes = to >= 0
    _close(ks[to[goes].cuda()], want[goes], bound[goes])
    assert torch.equal(vs.cpu()[to[goes]], v.cpu()[goes])
    kept = torch.ones(n_seq * room, dtype=torch.bool)
    kept[to[goes]] = False
    assert bool((ks.cpu()[kept] == 7).all()) and bool((vs.cpu()[kept] == 7).all())


def test_sine_and_cosine(ctx):
    """Of heads of ones with eps = 0 and a gradient of one in the first element of every pair, the weight's gradient is the cosine and less the sine of each
    pair's turn, and nothing else is rounded.  In 32 bits: the part of a quarter by which an angle is reduced is off by at most 2^-26, times pi / 2, and a polynomial's last
    two sums by 2^-25 each: below 2^-23."""
    rng = torch.Generator().manual_seed(0)
    D, worst = 128, 0.0
    edges = torch.tensor([0.0, 0.125, 0.25, 0.375, 0.5, 0.625, 0.75, 0.875, 1.0, 0.12500000001, 0.12499999999, 0.49999999999, 0.50000000001, 1e-9, 1e-4, 3.0], dtype=torch.float64)
    q = torch.ones(1, 1, D, dtype=BF16, device="cuda")
    d = torch.zeros_like(q)
    d[..., :D // 2] = 1
    for position in (1, -1, 2, 3, 1000, -12_345, (1 << 31) - 1, 1 << 40):
        for _ in range(4):
            turns = torch.cat([edges, torch.rand(D // 2 - len(edges), generator=rng, dtype=torch.float64)])
            _, _, dw, _ = ctx.norm_rotate_backward(d, d, q, q, None, None, turns.cuda(), eps=0.0, positions=torch.tensor([position]).cuda())
            whole = turns * position
            angle = (whole - whole.round()) * 2 * torch.pi
            worst = max(worst, float((dw.cpu().double() - torch.cat([angle.cos(), -angle.sin()])).abs().max()))
    assert worst <= 2.0 ** -23, worst


@pytest.mark.parametrize("exponent", [-60, -63, -64, -66, -69, 60])
def test_means_of_squares_that_are_denormal(ctx, exponent):
    """With no eps the smallest rows are of length one behind their norm too, as long as 32 bits hold their squares: 2^-138 has eleven of them, which is more
    than bfloat16 has."""
    H, D = 3, 16
    q = (1 + torch.rand(4, H, D, generator=torch.Generator().manual_seed(1))).to(BF16) * 2.0 ** exponent
    assert bool((q.double() * 2.0 ** -exponent >= 1).all())
    d = torch.randn(4, H, D, generator=torch.Generator().manual_seed(2)).to(BF16)
    there, position = torch.ones(4, dtype=torch.bool), torch.arange(4)
    turns = _turns(D)
    q_out, _ = ctx.norm_rotate(q.cuda(), q.cuda(), None, None, turns, eps=0.0)
    want, bound = rotate(q, torch.ones(D), turns.cpu(), position, there, 0.0, True)
    # the squares' own roundings, half a step of 2^-149 each, beside their mean
    denormal = 2.0 ** -150 / 4.0 ** exponent
    _close(q_out, want, bound + 2 * denormal * want.abs().amax())
    dq, _, dw, _ = ctx.norm_rotate_backward(d.cuda(), d.cuda(), q.cuda(), q.cuda(), None, None, turns, eps=0.0)
    dx, of_x, of_weight, of_bound = rotate_gradient(d, q, torch.ones(D), turns.cpu(), position, there, 0.0, True)
    _close(dq, dx, of_x + 8 * denormal * dx.abs().amax())
    assert bool(((dw.cpu().double() - of_weight).abs() <= 2.0 ** -24 * of_weight.abs() + of_bound + 8 * denormal * of_weight.abs().amax()).all())


# lengths of sequences; rows before the first and behind the last
RAGGED = [1, 0, 700, 3, 0, 0, 1500, 64, 65, 1, 1, 1900, 0, 333, 2, 5]


@pytest.mark.parametrize("heads,kv_heads,dim,turned", [(8, 8, 64, 64), (32, 8, 128, 128), (24, 16, 80, 32), (4, 2, 64, 64), (70, 5, 16, 16)])
@pytest.mark.parametrize("halves", [True, False])
def test_many_ragged_rows(ctx, heads, kv_heads, dim, turned, halves):
    """A wave takes all heads of a row, and many rows one after the other, across sequences' ends, empty ones among them, and rows of none; both directions, packed
    and, forward, into a store."""
    ptr = [5]
    for n in RAGGED * 2:
        ptr.append(ptr[-1] + n)
    rows = ptr[-1] + 9
    rng = torch.Generator(device="cuda").manual_seed(heads)
    x = (torch.randn(rows, heads + 2 * kv_heads, dim, generator=rng, device="cuda") * torch.exp(torch.randn(heads + 2 * kv_heads, 1, generator=rng, device="cuda"))).to(BF16)
    q, k, v = x.split([heads, kv_heads, kv_heads], dim=1)
    there, position, _ = places(rows, ptr)
    there, position = there.cuda(), position.cuda()
    for t in (q, k, v):
        t[~there] = float("nan")
    wq, wk = (1 + 0.3 * torch.randn(2, dim, generator=rng, device="cuda")).unbind()
    turns = _turns(turned)
    at = dict(q_ptr=torch.tensor(ptr).cuda(), halves=halves)
    q_out, k_out, v_out = ctx.norm_rotate(q, k, wq, wk, turns, v=v, **at)
    for got, t, w in ((q_out, q, wq), (k_out, k, wk)):
        _close(got, *rotate(t, w, turns, position, there, 1e-6, halves))
    assert torch.equal(v_out, torch.where(there[:, None, None], v, torch.zeros((), dtype=BF16, device="cuda")))
    d = [torch.randn(t.shape, generator=rng, device="cuda").to(BF16) for t in (q, k)]
    for t in d:
        t[~there] = float("nan")
    dq, dk, dwq, dwk = ctx.norm_rotate_backward(*d, q, k, wq, wk, turns, **at)
    for got, dw, t, w, back in ((dq, dwq, q, wq, d[0]), (dk, dwk, k, wk, d[1])):
        want, bound, of_weight, of_bound = rotate_gradient(back, t, w, turns, position, there, 1e-6, halves)
        _close(got, want, bound)
        # a lane adds up fewer than 64 terms here, some ten more sums join them, in the last ones' 64 bits; the terms' own errors as in tower_ref, with the sine's
        n = rows * t.shape[1]
        size = of_bound / (n * 2.0 ** -24 + (2 * dim + 32) * 2.0 ** -24 + TURN)
        assert bool(((dw.double() - of_weight).abs() <= 2.0 ** -24 * of_weight.abs() + ((80 + 2 * dim + 32) * 2.0 ** -24 + 2.0 ** -23) * size).all())
    # the same rows into a store, behind 3 of their sequence that were there
    past, room = 3, [n + 5 for n in RAGGED * 2]
    slots = [4]
    for n in room:
        slots.append(slots[-1] + n)
    used = torch.tensor([n + past for n in RAGGED * 2], dtype=torch.int32).cuda()
    ks, vs = (torch.full((slots[-1] + 2, kv_heads, dim), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    q_store, _, _ = ctx.norm_rotate(q, k, wq, wk, turns, v=v, k_ptr=torch.tensor(slots).cuda(), k_len=used, k_out=ks, v_out=vs, **at)
    there, position, to = places(rows, ptr, slots, used.tolist())
    goes = (to >= 0).cuda()
    assert torch.equal(goes, there.cuda())
    _close(q_store, *rotate(q, wq, turns, position.cuda(), there.cuda(), 1e-6, halves))
    want, bound = rotate(k, wk, turns, position.cuda(), there.cuda(), 1e-6, halves)
    _close(ks[to.cuda()[goes]], want[goes], bound[goes])
    assert torch.equal(vs[to.cuda()[goes]], v[goes])
    kept = torch.ones(len(ks), dtype=torch.bool, device="cuda")
    kept[to.cuda()[goes]] = False
    assert bool((ks[kept] == 7).all()) and bool((vs[kept] == 7).all())


@pytest.mark.parametrize("rows,heads,dim", [(1 << 21, 64, 128), (300_000, 3, 40)])
def test_long_sums_of_equal_terms(ctx, rows, heads, dim):
    """Heads of ones and the same gradient everywhere: the weight's gradient is that by sqrt(1 + eps), times rows and heads, of which each addition is rounded the same
    way.  At most 256 are added up behind one another, some 50 of such sums by a wave, and a few dozen more join those."""
    ones, d = torch.ones(1, 1, dim, dtype=BF16, device="cuda"), torch.linspace(0.1, 1.9, dim, device="cuda").to(BF16).view(1, 1, dim)
    q, k = ones.expand(rows, heads, dim), ones.expand(rows, 1, dim)
    _, _, dwq, dwk = ctx.norm_rotate_backward(d.expand(rows, heads, dim), d.expand(rows, 1, dim), q, k, None, None, None, eps=0.3)
    for dw, count in ((dwq, rows * heads), (dwk, rows)):
        want = d.double().flatten() * count / (1 + float(torch.tensor(0.3))) ** 0.5
        assert float(((dw.double() - want).abs() / want).max()) <= 400 * 2.0 ** -24, float(((dw.double() - want).abs() / want).max())
