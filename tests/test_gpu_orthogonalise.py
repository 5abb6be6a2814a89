"""Updates orthogonalised by Newton-Schulz products, against 64 bits (-m gpu).  Bounds: tower_ref.newton_schulz."""
import math

import pytest
import torch

from tower_ref import TINY, U, newton_schulz

pytestmark = pytest.mark.gpu

QUINTIC = (3.4445, -4.7750, 2.0315)
CUBIC = (1.5, -0.5, 0.0)


@pytest.fixture(scope="module")
def ctx():
    import paper_1806_11248_amd as g
    c = g.Context(0)
    yield c
    c.close()


def _matrix(m, n, seed, dtype=torch.float32, size=1e-3):
    rng = torch.Generator().manual_seed(seed)
    few = max(1, min(m, n) // 16)
    g = torch.randn(m, few, generator=rng) @ torch.randn(few, n, generator=rng) + torch.randn(m, n, generator=rng)
    return (g * size).to(dtype).cuda()


def _check(ctx, updates, steps=5, coefficients=QUINTIC, scales=1.0, outs=None):
    before = [u.cpu() for u in updates]
    lst = ctx.matrix_list(updates, outs, scales=scales)
    got = ctx.orthogonalise(lst, steps=steps, coefficients=coefficients)
    assert got is lst.outs
    for i, (o, g) in enumerate(zip(got, before)):
        scale = scales if isinstance(scales, float) else scales[i]
        want, bound = newton_schulz(g, steps, coefficients)
        if g.numel() == 0:
            continue
        err = o.cpu().double() - want * scale
        # the last rounding, and that of the product with the scale
        last = (U[o.dtype] + 2.0 ** -24) * float(torch.linalg.vector_norm(want * scale)) + TINY[o.dtype] * math.sqrt(o.numel())
        assert float(torch.linalg.vector_norm(err)) <= 1.001 * (abs(scale) * bound * (1 + U[o.dtype]) + last), (g.shape, float(torch.linalg.vector_norm(err)), bound, last)
        if outs is not None:
            assert torch.equal(updates[i].cpu(), g)
    return got


SHAPES = [(1, 1), (1, 9), (9, 1), (3, 5), (16, 16), (40, 64), (64, 256), (128, 64), (127, 129), (129, 127), (128, 128), (255, 384), (200, 1000), (1000, 200), (300, 300),
          (64, 64), (64, 384), (384, 64), (63, 383), (33, 31), (65, 64), (64, 385), (385, 17)]


@pytest.mark.parametrize("m,n", SHAPES)
@pytest.mark.parametrize("dtype", list(U))
def test_shapes(ctx, m, n, dtype):
    _check(ctx, [_matrix(m, n, m + n, dtype)])
    u = _matrix(m, n, m, dtype)
    _check(ctx, [u], outs=[torch.full_like(u, 9.0)], scales=0.2)


@pytest.mark.parametrize("steps,coefficients", [(1, QUINTIC), (2, QUINTIC), (3, QUINTIC), (10, QUINTIC), (8, CUBIC), (1, (1.0, 0.0, 0.0)), (4, (2.0, -1.5, 0.5))])
def test_steps_and_coefficients(ctx, steps, coefficients):
    _check(ctx, [_matrix(70, 150, 1), _matrix(64, 32, 2)], steps=steps, coefficients=coefficients)


def test_many_in_one_call(ctx):
    """Different shapes, types and scales, empty ones among them."""
    updates = [_matrix(m, n, i, list(U)[i % 3]) for i, (m, n) in enumerate(SHAPES + [(0, 5), (5, 0)] + [(7 * i % 90 + 1, 11 * i % 70 + 1) for i in range(1, 80)])]
    _check(ctx, updates, scales=[0.5 + 0.01 * i for i in range(len(updates))], outs=[torch.full_like(u, 9.0) for u in updates])
    assert ctx.orthogonalise(ctx.matrix_list([])) == []
    assert len(ctx.orthogonalise(ctx.matrix_list([torch.zeros(0, 3, device="cuda")]))) == 1


def test_equal_singular_values(ctx):
    """An orthogonal matrix: no error is taken on by much, so 22 bits and no fewer are seen."""
    q, _ = torch.linalg.qr(torch.randn(96, 96, generator=torch.Generator().manual_seed(1), dtype=torch.float64))
    u = q.float().contiguous().cuda()
    got = _check(ctx, [u.clone()])[0].cpu().double()
    t = 1 / math.sqrt(96)
    for _ in range(5):
        t *= QUINTIC[0] + QUINTIC[1] * t ** 2 + QUINTIC[2] * t ** 4
    assert float((got - t * q).abs().max()) < 2.0 ** -17 * t


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1.0, 1e15])
def test_the_size_of_an_update_does_not_matter(ctx, size):
    u = _matrix(50, 90, 3, size=1.0)
    one = ctx.orthogonalise(ctx.matrix_list([u], [torch.zeros_like(u)]))[0]
    power = 2.0 ** round(math.log2(size))
    other = ctx.orthogonalise(ctx.matrix_list([u * power], [torch.zeros_like(u)]))[0]
    assert torch.equal(one, other)


def test_zeros_low_rank_and_what_is_not_finite(ctx):
    zero, nan, inf, fine = torch.zeros(40, 70, device="cuda"), _matrix(40, 70, 1), _matrix(70, 40, 2), _matrix(40, 70, 3)
    nan[3, 4], inf[5, 6] = math.nan, -math.inf
    rank_one = torch.outer(torch.arange(1.0, 31.0), torch.arange(1.0, 91.0)).cuda()
    row = torch.zeros(20, 60, device="cuda")
    row[7, 9] = -3.0
    alone = ctx.orthogonalise(ctx.matrix_list([fine], [torch.zeros_like(fine)]))[0]
    outs = [torch.full_like(t, 9.0) for t in (zero, nan, inf, fine, row)]
    ctx.orthogonalise(ctx.matrix_list([zero, nan, inf, fine, row], outs))
    assert bool((outs[0] == 0).all()) and bool(outs[1].isnan().all()) and bool(outs[2].isnan().all()) and torch.equal(outs[3], alone)
    want, bound = newton_schulz(row.cpu(), 5, QUINTIC)
    assert abs(float(outs[4][7, 9]) - float(want[7, 9])) <= bound and int((outs[4] != 0).sum()) == 1
    got = ctx.orthogonalise(ctx.matrix_list([rank_one.clone()]))[0].cpu().double()
    # one singular value; the others are what rounding leaves of zero, which the steps multiply by 3.4445 each
    s = torch.linalg.svdvals(got)
    assert abs(float(s[0]) - float(torch.linalg.svdvals(newton_schulz(rank_one.cpu()[:1, :1], 5, QUINTIC)[0])[0])) < 1e-4 and float(s[1]) < 3.4445 ** 5 * 2.0 ** -21


def test_the_same_alone_together_and_on_every_run(ctx):
    updates = [_matrix(m, n, i) for i, (m, n) in enumerate([(200, 333), (64, 64), (500, 130), (30, 700)])]
    alone = [ctx.orthogonalise(ctx.matrix_list([u], [torch.zeros_like(u)]))[0] for u in updates]
    outs = [torch.zeros_like(u) for u in updates]
    lst = ctx.matrix_list(updates, outs)
    for _ in range(3):
        ctx.orthogonalise(lst)
        assert all(torch.equal(a, b) for a, b in zip(alone, outs))
    for u in updates:
        u.mul_(2.0)                                                             # new values in the same places
    ctx.orthogonalise(lst)
    assert all(torch.equal(a, b) for a, b in zip(alone, outs))
    for u in updates:
        u.neg_()                                                                # (sums in the matrix units need not round both signs alike)
    ctx.orthogonalise(lst)
    for a, b, u in zip(alone, outs, updates):
        assert float(torch.linalg.vector_norm(a.double() + b.double())) <= 2 * newton_schulz(u.cpu(), 5, QUINTIC)[1]


def test_parts_of_a_buffer(ctx):
    """Matrices that begin anywhere; what lies before and behind stays."""
    for dtype in U:
        flat = torch.randn(5000, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
        for shift in (1, 3):
            keep = flat.clone()
            part = keep[shift:shift + 33 * 47].view(33, 47)
            _check(ctx, [part])
            assert torch.equal(keep[:shift], flat[:shift]) and torch.equal(keep[shift + 33 * 47:], flat[shift + 33 * 47:])


@pytest.mark.parametrize("m,n", [(72, 100), (100, 72), (70, 99), (99, 70), (132, 66), (66, 132)])
def test_parts_of_a_buffer_by_several_workgroups(ctx, m, n):
    """Results that can be written by fours, and those that cannot, for their columns or for where they begin."""
    for dtype in U:
        flat = torch.randn(m * n + 16, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
        for shift in (0, 1, 2, 4, 8):
            keep = flat.clone()
            _check(ctx, [keep[shift:shift + m * n].view(m, n)])
            assert torch.equal(keep[:shift], flat[:shift]) and torch.equal(keep[shift + m * n:], flat[shift + m * n:])


def test_in_a_graph():
    import paper_1806_11248_amd as g
    side = torch.cuda.Stream()
    own = g.Context(0, stream=side)
    try:
        updates = [_matrix(130, 70, 1), _matrix(40, 64, 2, torch.bfloat16)]
        outs = [torch.zeros_like(u) for u in updates]
        side.wait_stream(torch.cuda.current_stream())
        lst = own.matrix_list(updates, outs)
        with torch.cuda.stream(side):
            own.orthogonalise(lst)
            side.synchronize()
            graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
            for graph in graphs:
                with torch.cuda.graph(graph, stream=side):
                    own.orthogonalise(lst)
            for step in range(3):
                for u in updates:
                    u.copy_(torch.randn(u.shape, generator=torch.Generator().manual_seed(step)))
                own.orthogonalise(lst)
                side.synchronize()
                want = [o.clone() for o in outs]
                for graph in graphs:
                    for o in outs:
                        o.zero_()
                    graph.replay()
                    side.synchronize()
                    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    finally:
        own.close()


def test_a_list_keeps_its_memory(ctx):
    t, o = _matrix(40, 50, 1), torch.zeros(40, 50, device="cuda")
    want = ctx.orthogonalise(ctx.matrix_list([t], [torch.zeros_like(t)]))[0]
    places = t.data_ptr(), o.data_ptr()
    held = o.view(40, 50)
    lst = ctx.matrix_list([t], [o])
    t.data, o.data = torch.full((40, 50), 5.0, device="cuda"), torch.full((40, 50), 6.0, device="cuda")
    others = [torch.full((40, 50), 9.0, device="cuda") for _ in range(8)]
    assert not {x.data_ptr() for x in [t, o, *others]} & set(places)
    ctx.orthogonalise(lst)
    assert torch.equal(held, want) and bool((o == 6.0).all()) and all(bool((x == 9.0).all()) for x in others)


def test_results_over_one_another_are_refused(ctx):
    import paper_1806_11248_amd as g
    flat = torch.ones(4000, device="cuda")
    a, b, near = flat[:1000].view(20, 50), flat[1000:2000].view(20, 50), flat[980:1980].view(20, 50)
    for tensors, outs in (([a, a], [a, a]), ([a, b], [b, a]), ([a, b], [near, b]), ([near], [b]), ([a, b], [flat[2000:3000].view(20, 50), flat[2999:3999].view(20, 50)]),
                          ([b, a, near], [b, flat[2000:3000].view(20, 50), flat[3000:].view(20, 50)])):
        with pytest.raises(g.GbtError) as e:
            ctx.matrix_list(tensors, outs)
        assert e.value.code == g.binding.EINVAL
    # the same matrix read by two, and neighbours
    ctx.matrix_list([a, a, near], [flat[2000:3000].view(20, 50), flat[3000:].view(20, 50), torch.ones_like(near)])
    ctx.matrix_list([a, b])
    assert bool((flat == 1).all())


def test_refusals(ctx):
    import paper_1806_11248_amd as g
    t = torch.ones(10, 10, device="cuda")
    for call in (lambda: ctx.matrix_list([t.double()]), lambda: ctx.matrix_list([t[0]]), lambda: ctx.matrix_list([t.cpu()]), lambda: ctx.matrix_list([t[:, :5]]),
                 lambda: ctx.matrix_list([t], [t[:5]]), lambda: ctx.matrix_list([t], []), lambda: ctx.matrix_list([t], scales=[1.0, 2.0]),
                 lambda: ctx.matrix_list([t], [t.half()])):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(g.GbtError):
        ctx.matrix_list([t], scales=math.inf)
    lst = ctx.matrix_list([t])
    for kw in (dict(steps=0), dict(steps=33), dict(coefficients=(math.nan, 0.0, 0.0)), dict(coefficients=(5.0, 0.0, 0.0)), dict(coefficients=(3.4445, -4.775, 20.0))):
        with pytest.raises(g.GbtError) as e:
            ctx.orthogonalise(lst, **kw)
        assert e.value.code == g.binding.EINVAL
    assert bool((t == 1).all())
