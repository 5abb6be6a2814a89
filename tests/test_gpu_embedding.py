"""Rows of an embedding table and the table's gradient, against 64-bit sums (-m gpu).

A looked-up element is one product in 32 bits and one rounding; a gradient is a sum in 32 bits, whose error no order makes larger than that of n - 1
roundings of partial sums, one product, and one rounding.
"""
import math

import pytest
import torch

from tower_ref import TINY, U, U32, lookup_gradient

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    import paper_1806_11248_amd as g
    c = g.Context(0)
    yield c
    c.close()


def _ids(places, rows, seed, outside=True, wide=True, skew=1.0):
    rng = torch.Generator().manual_seed(seed)
    ids = (rows * torch.rand(places, generator=rng) ** (1 + skew)).long().clamp_max(rows - 1)
    if outside and places > 3:
        ids[torch.randperm(places, generator=rng)[:max(1, places // 17)]] = -1
        ids[0], ids[-1] = rows, (1 << 40) + 1 if wide else -(1 << 31)
    return ids if wide else ids.int()


def _close(got, want, bound=0.0):
    want = want.to(got.device)
    bound = bound.to(got.device) if isinstance(bound, torch.Tensor) else bound
    err = (got.double() - want).abs()
    tol = 1.001 * (U[got.dtype] * want.abs() + (1 + U[got.dtype]) * bound) + TINY[got.dtype]
    assert bool((err <= tol).all()), float((err - tol).max())


def _check_lookup(ctx, table, ids, scale, dtype=None, out=None):
    got = ctx.embedding(table, ids.cuda(), scale=scale, dtype=dtype, out=out)
    rows = table.shape[0]
    flat = ids.flatten().long()
    inside = (flat >= 0) & (flat < rows)
    want = torch.zeros(len(flat), table.shape[1], dtype=torch.float64)
    if rows:
        want[inside] = table.cpu().double()[flat[inside]] * scale
    _close(got.reshape(want.shape), want, U32 * want.abs())
    assert bool((got.reshape(want.shape).cpu()[~inside] == 0).all())
    return got


def _check_gradient(ctx, dout, ids, rows, scale, dtype=F32, out=None, accumulate=False):
    old = out.cpu() if accumulate else None
    want, bound = lookup_gradient(dout.cpu(), ids, rows, scale, old)
    got = ctx.embedding_backward(dout, ids.cuda(), rows, scale=scale, dtype=dtype, out=out, accumulate=accumulate)
    _close(got, want, bound)
    flat = ids.flatten().long()
    untouched = torch.ones(rows, dtype=torch.bool)
    untouched[flat[(flat >= 0) & (flat < rows)]] = False
    assert torch.equal(got.cpu()[untouched], old[untouched] if accumulate else torch.zeros_like(got.cpu()[untouched]))
    return got


@pytest.mark.parametrize("places,rows,width", [(1, 1, 8), (1, 7, 1), (3, 5, 3), (48, 500, 512), (63, 9, 520), (257, 40, 77), (1000, 3, 64), (5000, 700, 24),
                                               (70_001, 12, 16), (9, 11, 4104)])
@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F32, BF16), (F16, F32), (BF16, F16)])
def test_lookup(ctx, places, rows, width, types):
    rng = torch.Generator().manual_seed(places)
    table = torch.randn(rows, width, generator=rng).to(types[0]).cuda()
    for wide in (False, True):
        _check_lookup(ctx, table, _ids(places, rows, width, wide=wide), math.sqrt(width), types[1])


# few ids, up to the last number of them that are not sorted and the first that are; many; one or two passes of digits, or three; chunks that end inside runs
SIZES = [(1, 1, 8), (2, 5, 1), (33, 9, 24), (1999, 40, 64), (2048, 3, 100), (2048, 5000, 16), (2049, 3, 100), (2049, 5000, 16), (4097, 1, 8), (9_000, 1023, 33),
         (9_000, 1024, 40), (20_000, 12, 64), (12_289, 70_000, 12), (8_193, 2_000_000, 3), (5_000, 600, 1032),
         # the most rows and columns that are added up in LDS, one more; groups of lanes that have no place
         (30_000, 32, 24), (30_000, 33, 24), (2_500, 31, 1), (5_000, 7, 256), (3_000, 32, 250), (3_000, 32, 257), (2_049, 32, 8), (100_003, 12, 64), (5_000, 7, 1032)]


@pytest.mark.parametrize("places,rows,width", SIZES)
@pytest.mark.parametrize("types", [(F32, F32), (BF16, F32), (F16, F16), (BF16, BF16)])
def test_gradient(ctx, places, rows, width, types):
    rng = torch.Generator().manual_seed(rows)
    dout = torch.randn(places, width, generator=rng).to(types[0]).cuda()
    for wide, skew in ((True, 1.0), (False, 4.0)):
        _check_gradient(ctx, dout, _ids(places, rows, places, wide=wide, skew=skew), rows, 1.7, types[1])


@pytest.mark.parametrize("places,rows", [(2000, 30), (2000, 5000), (30_000, 30), (30_000, 5000)])
def test_accumulate(ctx, places, rows):
    """Added to what is there; rows without an id stay as they are, whatever they hold."""
    for dtype in U:
        dout = torch.randn(places, 40, generator=torch.Generator().manual_seed(1)).cuda()
        out = torch.randn(rows, 40, generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
        _check_gradient(ctx, dout, _ids(places, rows, 5), rows, 0.5, out=out, accumulate=True)
    out = torch.full((rows, 40), math.nan, device="cuda")
    ctx.embedding_backward(dout, torch.full((places,), 3, device="cuda"), rows, out=out, accumulate=True)
    assert bool(out.isnan().all())
    out.fill_(math.inf)
    ctx.embedding_backward(dout, torch.full((places,), -1, device="cuda"), rows, out=out, accumulate=True)
    assert bool((out == math.inf).all())


@pytest.mark.parametrize("places", [1500, 50_000])
def test_one_id_everywhere_and_none_inside(ctx, places):
    """Runs over all chunks, and lists of which nothing is left."""
    dout = torch.randn(places, 72, generator=torch.Generator().manual_seed(1)).cuda()
    for rows in (1, 100, 3000):
        for v in (0, rows - 1):
            _check_gradient(ctx, dout, torch.full((places,), v), rows, 1.0)
        _check_gradient(ctx, dout, torch.full((places,), rows), rows, 1.0)
        _check_gradient(ctx, dout, torch.cat([torch.full((places - 1,), rows - 1), torch.tensor([0])]), rows, 1.0)


def test_shapes_strides_and_alignment(ctx):
    """Ids of any shape, rows any distance apart, parts of a wider tensor that do not begin at 16 bytes, expanded gradients."""
    rng = torch.Generator().manual_seed(0)
    ids = _ids(24, 50, 3).view(2, 3, 4)
    table = torch.randn(50, 100, generator=rng).cuda()
    for lo, hi in ((0, 64), (8, 72), (1, 65), (4, 100), (99, 100)):
        got = _check_lookup(ctx, table[:, lo:hi], ids, 2.0)
        assert got.shape == (2, 3, 4, hi - lo)
        out = torch.full((24, 120), 7.0, device="cuda")
        _check_lookup(ctx, table[:, lo:hi], ids, 2.0, out=out[:, 5:5 + hi - lo])
        assert bool((out[:, :5] == 7).all()) and bool((out[:, 5 + hi - lo:] == 7).all())
        for places in (24, 4000):
            many = ids.flatten() if places == 24 else _ids(places, 50, 4)
            dout = torch.randn(places, 100, generator=rng).cuda()[:, lo:hi]
            grad = torch.full((50, 120), 7.0, device="cuda")
            _check_gradient(ctx, dout, many, 50, 1.0, out=grad[:, 5:5 + hi - lo])
            assert bool((grad[:, :5] == 7).all()) and bool((grad[:, 5 + hi - lo:] == 7).all())
    dout = torch.randn(1, 64, generator=rng).cuda().expand(5000, 64)          # the same gradient for every place
    _check_gradient(ctx, dout, _ids(5000, 50, 6), 50, 1.0)
    one = torch.randn(64, generator=rng).cuda().expand(50, 64)                # the same row for every id
    _check_lookup(ctx, one, ids, 1.0)
    shaped = torch.randn(2, 3, 4, 16, generator=rng).cuda()
    _check_gradient(ctx, shaped, ids, 50, 1.0)
    same = torch.arange(6, device="cuda").view(2, 3)
    assert torch.equal(ctx.embedding(table, same), ctx.embedding(table, same.flatten()).view(2, 3, 100))


def test_empty(ctx):
    table = torch.randn(5, 16, device="cuda")
    none = torch.zeros(0, dtype=torch.int64)
    assert ctx.embedding(table, none.cuda()).shape == (0, 16)
    _check_lookup(ctx, table[:0], torch.tensor([0, -1, 3]), 1.0)
    assert bool((ctx.embedding_backward(table[:0], none.cuda(), 5) == 0).all())
    assert bool((ctx.embedding_backward(table[:0, :3], none.cuda(), 200_000) == 0).all())
    assert ctx.embedding_backward(table, torch.arange(5, device="cuda"), 0).shape == (0, 16)
    out = torch.ones(5, 16, device="cuda")
    assert bool((ctx.embedding_backward(table[:0], none.cuda(), out=out, accumulate=True) == 1).all())


def test_what_is_not_finite_stays_in_its_row(ctx):
    for places in (1000, 20_000):
        ids = torch.arange(places) % 100
        dout = torch.randn(places, 24, generator=torch.Generator().manual_seed(1)).cuda()
        dout[7] = math.nan
        dout[8, 3] = math.inf
        got = ctx.embedding_backward(dout, ids.cuda(), 100)
        assert bool(got[7].isnan().all()) and bool((got[8, 3] == math.inf)) and bool(got[9:].isfinite().all()) and bool(got[:7].isfinite().all())
        ids[7] = ids[8] = -1                                                   # padded places do not count
        assert bool(ctx.embedding_backward(dout, ids.cuda(), 100).isfinite().all())


@pytest.mark.parametrize("places,rows", [(2000, 40), (60_000, 40), (60_000, 9_000)])
def test_the_same_on_every_run(ctx, places, rows):
    dout, ids = torch.randn(places, 56, device="cuda"), _ids(places, rows, 2).cuda()
    first = ctx.embedding_backward(dout, ids, rows)
    for _ in range(3):
        torch.randn(1 << 20, device="cuda")
        assert torch.equal(ctx.embedding_backward(dout, ids, rows), first)


def test_a_gradient_against_differences(ctx):
    """The loss is a weighted sum of what is looked up; a step along each row changes it by the gradient."""
    ids = _ids(300, 20, 1)
    table = torch.randint(-8, 9, (20, 16), generator=torch.Generator().manual_seed(1)).float().cuda()
    dout = torch.randint(-8, 9, (300, 16), generator=torch.Generator().manual_seed(2)).float().cuda()
    grad = ctx.embedding_backward(dout, ids.cuda(), 20, scale=0.5)

    def loss(t):
        return float((ctx.embedding(t, ids.cuda(), scale=0.5).double() * dout.double()).sum())

    for v in range(20):
        for e in (0, 15):
            step = torch.zeros_like(table)
            step[v, e] = 1.0
            assert loss(table + step) - loss(table - step) == 2 * float(grad[v, e])    # whole numbers and halves: exact


@pytest.mark.parametrize("places", [500, 30_000])
def test_in_graphs(places):
    """Captured with the ids in a buffer of their own, replayed with others, between eager calls that use the context's workspace."""
    import paper_1806_11248_amd as g
    side = torch.cuda.Stream()
    own = g.Context(0, stream=side)
    try:
        table = torch.randn(300, 48, device="cuda")
        dout, ids = torch.randn(places, 48, device="cuda"), _ids(places, 300, 0).cuda()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            own.embedding(table, ids), own.embedding_backward(dout, ids, 300)
            side.synchronize()
            graphs = []
            for _ in range(2):
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    both = own.embedding(table, ids), own.embedding_backward(dout, ids, 300)
                graphs.append((graph, both))
            for step in range(4):
                ids.copy_(_ids(places, 300, 10 + step))
                for graph, both in graphs:
                    graph.replay()
                eager = own.embedding(table, ids), own.embedding_backward(dout, ids, 300)
                side.synchronize()
                for graph, both in graphs:
                    assert all(torch.equal(a, b) for a, b in zip(both, eager))
    finally:
        own.close()


def test_another_stream(ctx):
    """A context on a stream of its own, called while torch works on another: outputs are the context's, and the inputs' memory stays until it is done."""
    import paper_1806_11248_amd as g
    side = torch.cuda.Stream()
    own = g.Context(0, stream=side)
    try:
        table, ids = torch.randn(1000, 64, device="cuda"), _ids(20_000, 1000, 0).cuda()
        dout = torch.randn(20_000, 64, device="cuda")
        want = ctx.embedding(table, ids), ctx.embedding_backward(dout, ids, 1000)
        torch.cuda.synchronize()
        for _ in range(3):
            t, d = table.clone(), dout.clone()
            side.wait_stream(torch.cuda.current_stream())
            got = own.embedding(t, ids), own.embedding_backward(d, ids, 1000)
            del t, d
            others = [torch.full_like(dout, 9.0) for _ in range(4)]
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)) and len(others) == 4
    finally:
        own.close()


def test_a_gradient_that_has_to_be_copied_on_another_stream():
    """A gradient of three axes that no view makes two of: its copy is the context's stream's work too, so what torch's own stream is busy with does not delay it."""
    import paper_1806_11248_amd as g
    side = torch.cuda.Stream()
    own = g.Context(0, stream=side)
    try:
        ids = _ids(2000, 30, 0).view(50, 40).cuda()
        dout = torch.randn(40, 50, 3, 64, device="cuda")[:, :, 1].transpose(0, 1)
        whole, a = dout.contiguous(), torch.randn(4096, 4096, device="cuda")
        torch.cuda.synchronize()
        want = own.embedding_backward(whole, ids, 30)
        side.synchronize()
        for _ in range(20):
            a = a @ a * 1e-4
        got = own.embedding_backward(dout, ids, 30)
        side.synchronize()
        assert torch.equal(got, want)
    finally:
        own.close()


def test_refusals(ctx):
    import paper_1806_11248_amd as g
    table, ids = torch.randn(5, 16, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    for call in (lambda: ctx.embedding(table.double(), ids), lambda: ctx.embedding(table.cpu(), ids), lambda: ctx.embedding(table, ids.cpu()),
                 lambda: ctx.embedding(table, ids.float()), lambda: ctx.embedding(table, ids.repeat(2)[::2]), lambda: ctx.embedding(table[0], ids),
                 lambda: ctx.embedding(table.t(), ids), lambda: ctx.embedding(table, ids, dtype=torch.float64), lambda: ctx.embedding(table, ids, out=table[:2]),
                 lambda: ctx.embedding(table, ids, out=table[:3], dtype=torch.bfloat16), lambda: ctx.embedding_backward(table, ids, 5),
                 lambda: ctx.embedding_backward(table[:3], ids), lambda: ctx.embedding_backward(table[:3], ids, 5, accumulate=True),
                 lambda: ctx.embedding_backward(table[:3], ids, 5, out=table[:4]), lambda: ctx.embedding_backward(table[:3], ids, 5, dtype=torch.int32),
                 lambda: ctx.embedding_backward(table[:3].double(), ids, 5)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: ctx.embedding(table, ids, scale=math.inf), lambda: ctx.embedding(table, ids, out=table[:1].expand(3, 16)),
                 lambda: ctx.embedding_backward(table[:3], ids, 5, scale=math.nan), lambda: ctx.embedding_backward(table[:3], ids, out=table[:1].expand(5, 16))):
        with pytest.raises(g.GbtError) as e:
            call()
        assert e.value.code == g.binding.EINVAL
