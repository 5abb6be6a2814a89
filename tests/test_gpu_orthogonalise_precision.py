"""How exact orthogonalised updates are: beside the same formulas in 32-bit products (-m gpu).

Errors are against 64 bits.  What float32 results may be off by is three times what 32-bit products are, on the same matrix; nothing in the formulas says which
of two ways to round is ahead, and the two differ by their operands (22 bits in place of 24) and by the order of their sums.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

QUINTIC = (3.4445, -4.7750, 2.0315)
TIMES = 3.0


@pytest.fixture(scope="module")
def ctx():
    import paper_1806_11248_amd as g
    c = g.Context(0)
    yield c
    c.close()


def exact(g, steps=5, coefficients=QUINTIC):
    """In 64 bits, by the polynomial of X X^T that all steps together are."""
    a, b, c = coefficients
    x = g.double() / torch.linalg.vector_norm(g.double())
    x = x.t().contiguous() if g.shape[0] > g.shape[1] else x
    gram = x @ x.t().contiguous()
    eye = torch.eye(len(gram), dtype=torch.float64, device=g.device)
    total = eye
    for _ in range(steps):
        factor = a * eye + b * gram + c * (gram @ gram)
        total, gram = factor @ total, factor @ gram @ factor
    return (total @ x).t() if g.shape[0] > g.shape[1] else total @ x


def in_32_bits(g, steps=5, coefficients=QUINTIC):
    a, b, c = coefficients
    x = (g.double() / torch.linalg.vector_norm(g.double())).float()
    x = x.t().contiguous() if g.shape[0] > g.shape[1] else x
    for _ in range(steps):
        gram = x @ x.t().contiguous()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.t() if g.shape[0] > g.shape[1] else x


def off(x, want):
    return float(torch.linalg.vector_norm(x.double() - want))


def off_by_row(x, want):
    """Of each row, relative to its length."""
    return torch.linalg.vector_norm(x.double() - want, dim=1) / torch.linalg.vector_norm(want, dim=1)


@pytest.mark.parametrize("m,n", [(64, 256), (40, 300), (200, 700), (512, 2048), (900, 1000)])
@pytest.mark.parametrize("spread", [1e-4, 1e-6])
@pytest.mark.parametrize("steps", [5, 10])
def test_rows_of_very_different_size(ctx, m, n, spread, steps):
    """Rarely used rows of a matrix.  X's elements are held with an error of at most 2^-39 (of a bound between 1 and 2, twice 2^-40), factors with one
    of 2^-38, of which a row takes the length of a row times X's largest singular value, below 1.2: of a row of length r, their share is (2^-39 sqrt n + 1.2 * 2^-38 sqrt m) / r, in the
    first step, of which all are at most 1.5 times as much, as such rows grow by 3.4445 in each.

    Rows are compared that have not left the length of a tenth behind the last step (r * 3.4445 ** steps <= 0.1).  A step multiplies those by 3.4445 - 4.775 t^2 for
    a t of at most a tenth, and an error of them by 3.4445 - 3 * 4.775 t^2, so what they are off by stays what it was, relative to them, but for one part in
    ten.  A longer one's error is multiplied in every step by the polynomial's slope where it lies, which is between -1.7 and 4.3, while its length stays around one: by ten
    steps one row of hundreds is off by 16 times what its neighbours are, on either side, and the quotient of two such errors is that of two single roundings, of
    any size.  For all rows together their lengths' root mean square is compared, in which no single row counts."""
    rng = torch.Generator().manual_seed(m)
    g = torch.randn(m, n, generator=rng) * torch.logspace(0, math.log10(spread), m)[:, None]
    want, other = exact(g, steps), in_32_bits(g, steps)
    for tall in (False, True):
        u = (g.t().contiguous() if tall else g).cuda()
        got = ctx.orthogonalise(ctx.matrix_list([u], [torch.zeros_like(u)]), steps=steps)[0].cpu()
        got = got.t() if tall else got
        assert off(got, want) <= TIMES * off(other, want)
        r = torch.linalg.vector_norm(g.double(), dim=1) / torch.linalg.vector_norm(g.double())
        held = 1.5 * (2.0 ** -39 * math.sqrt(n) + 1.2 * 2.0 ** -38 * math.sqrt(m)) / r
        short = r * 3.4445 ** steps <= 0.1
        if bool(short.any()):
            assert bool((off_by_row(got, want)[short] <= TIMES * off_by_row(other, want)[short].max() + held[short]).all())


@pytest.mark.parametrize("steps,factor", [(1, 0.1), (3, 0.1), (4, 0.02)])
def test_factors_far_below_one(ctx, steps, factor):
    """Singular values that shrink with every step are held with what they have then."""
    for m, n in ((40, 64), (130, 150)):
        for dtype in (torch.float32, torch.bfloat16):
            g = torch.randn(m, n, generator=torch.Generator().manual_seed(1)).to(dtype)
            u = g.cuda()
            got = ctx.orthogonalise(ctx.matrix_list([u]), steps=steps, coefficients=(factor, 0.0, 0.0))[0].cpu()
            want = exact(g, steps, (factor, 0.0, 0.0))
            # a rounding of 22 bits for each of three products a step at most, sums in 32 bits, and the result's
            assert off(got, want) <= (steps * 6 * 2.0 ** -22 + torch.finfo(dtype).eps / 2) * float(torch.linalg.vector_norm(want))


def _averaged(m, n, seed, dtype=torch.float32):
    """A few strong directions, and many weak ones."""
    rng = torch.Generator(device="cuda").manual_seed(seed)
    few = max(1, min(m, n) // 16)
    g = torch.randn(m, few, generator=rng, device="cuda") @ torch.randn(few, n, generator=rng, device="cuda") + torch.randn(m, n, generator=rng, device="cuda")
    return g.to(dtype)


# one workgroup's; one tile; one step on A at a time, several tiles; two steps; rows of tiles past the first eight; more tiles than run at once
SHAPES = [(64, 64), (64, 256), (384, 40), (100, 120), (128, 128), (200, 1500), (300, 300), (1500, 200), (400, 400), (512, 2048), (700, 2400), (767, 800), (768, 768), (777, 1001),
          (1001, 777), (900, 900), (1100, 1400), (2100, 4200), (4200, 2100),
          # a few long rows
          (689, 15), (30, 2000), (12, 1108), (20, 300), (8, 380), (1000, 8)]


@pytest.mark.parametrize("m,n", SHAPES)
def test_as_exact_as_32_bit_products(ctx, m, n):
    """Beside the library's on this card: a quarter more at most, for what errors of one matrix differ from those of the next.  Operands of one part would be off
    a thousand times as far."""
    count = max(1, min(24, 200_000 // (m * n)))
    updates = [_averaged(m, n, seed) for seed in range(count)]
    outs = ctx.orthogonalise(ctx.matrix_list(updates, [torch.zeros_like(u) for u in updates]))
    want = [exact(u) for u in updates]
    here = math.sqrt(sum(off(o, w) ** 2 for o, w in zip(outs, want)))
    there = math.sqrt(sum(off(in_32_bits(u), w) ** 2 for u, w in zip(updates, want)))
    assert here <= 1.25 * there, (here, there)


@pytest.mark.parametrize("m,n", [s for s in SHAPES if max(s) < 2100])
def test_sixteen_bit_results_are_rounded_ones(ctx, m, n):
    """A result of sixteen bits hides an error before its last rounding, except where that lands on the other side of a middle: the share of such elements is the
    error's mean size by the distance of two numbers.  It is at most three times that of 32-bit products (TIMES), and four standard deviations of a count."""
    for dtype in (torch.float16, torch.bfloat16):
        count = max(1, min(24, 400_000 // (m * n)))
        updates = [_averaged(m, n, seed, dtype) for seed in range(count)]
        outs = ctx.orthogonalise(ctx.matrix_list(updates, [torch.zeros_like(u) for u in updates]))
        want = [exact(u).to(dtype) for u in updates]
        here = sum(int((o != w).sum()) for o, w in zip(outs, want))
        there = sum(int((in_32_bits(u).to(dtype) != w).sum()) for u, w in zip(updates, want))
        assert here <= TIMES * there + 4 * math.sqrt(TIMES * there + 1), (here, there, count * m * n)


def _check_list(ctx, updates):
    """Float32 results beside 32-bit products, all of a shape together; those of sixteen bits by the share that is not the rounded 64-bit one."""
    scales = [0.5 + 0.25 * (i % 3) for i in range(len(updates))]                     # what they are multiplied by is exact in each type
    outs = ctx.orthogonalise(ctx.matrix_list(updates, [torch.full_like(u, 9.0) for u in updates], scales=scales))
    for u, o, scale in zip(updates, outs, scales):
        want, other = exact(u) * scale, in_32_bits(u) * scale
        if u.dtype is torch.float32:
            assert off(o, want) <= 1.25 * off(other, want), (u.shape, off(o, want), off(other, want))
        else:
            here, there = (int((x.to(u.dtype) != want.to(u.dtype)).sum()) for x in (o, other))
            assert here <= TIMES * there + 4 * math.sqrt(TIMES * there + 1), (u.shape, u.dtype, here, there)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_more_tiles_than_run_at_once(ctx, dtype):
    """Symmetric products of more than 512 tiles too, two workgroups on a compute unit: 8 x 45 and 8 x 28 of them, and 16 x 10, wide and tall, with odd sizes."""
    _check_list(ctx, [_averaged(m, n, seed, dtype) for seed in range(8) for m, n in ((1100, 1400), (1001, 777), (512, 2048), (2048, 512))])


def test_all_kinds_in_one_list(ctx):
    """Kinds one after the other, of which each begins with the first tile of its own."""
    shapes = [(64, 200), (300, 500), (1100, 900), (200, 1700), (2200, 1300), (40, 40), (129, 1000)]
    _check_list(ctx, [_averaged(m, n, 100 + i, dtype) for i, (m, n) in enumerate(shapes) for dtype in (torch.bfloat16, torch.float32, torch.float16)])


def test_groups_that_share_the_workspace(ctx):
    """Matrices of 1.6 GB of workspace each are worked on one after the other, in the same memory; the longest rows that there can be."""
    updates = [_averaged(128, 1 << 20, 1, torch.bfloat16), _averaged(1 << 20, 100, 2, torch.bfloat16), _averaged(90, 70, 3, torch.bfloat16)]
    lst = ctx.matrix_list(updates, [torch.zeros_like(u) for u in updates])
    assert (3 << 29) < lst.workspace_bytes <= (2 << 30)
    outs = ctx.orthogonalise(lst)
    for u, o in zip(updates, outs):
        want = exact(u).to(u.dtype)
        here, there = int((o != want).sum()), int((in_32_bits(u).to(u.dtype) != want).sum())
        assert here <= TIMES * there + 4 * math.sqrt(TIMES * there + 1), (u.shape, here, there)


@pytest.mark.parametrize("steps", [3, 4, 8, 13])
@pytest.mark.parametrize("coefficients", [(1.5, -0.5, 0.0), (1.875, -1.25, 0.375)])
def test_factors_of_less_than_two(ctx, steps, coefficients):
    """Iterations that end at one without going past it: x f(x) has a slope between zero and f(x), so no step makes a relative error larger, and 32-bit products
    are off by a few roundings in all.  Results here are off by those of 22 bits and a sign, 2^-23, of X, of F, of what A adds to F (less than F itself is), and by low * low,
    which is left out and is as much: four of them a step at most."""
    for m, n, dtype in ((40, 64, torch.float16), (130, 150, torch.float16), (300, 500, torch.float16), (800, 900, torch.float32), (70, 150, torch.float32), (40, 30, torch.float32)):
        updates = [_averaged(m, n, seed, dtype) for seed in range(max(1, min(8, 100_000 // (m * n))))]
        outs = ctx.orthogonalise(ctx.matrix_list(updates, [torch.zeros_like(u) for u in updates]), steps=steps, coefficients=coefficients)
        want, others = [exact(u, steps, coefficients) for u in updates], [in_32_bits(u, steps, coefficients) for u in updates]
        if dtype is torch.float32:
            here, there = (math.sqrt(sum(off(o, w) ** 2 for o, w in zip(x, want))) for x in (outs, others))
            length = math.sqrt(sum(float(torch.linalg.vector_norm(w)) ** 2 for w in want))
            assert here <= max(TIMES * there, 4 * steps * 2.0 ** -23 * length), (m, n, here, there, length)
        else:
            here, there = (sum(int((o.to(dtype) != w.to(dtype)).sum()) for o, w in zip(x, want)) for x in (outs, others))
            assert here <= TIMES * there + 4 * math.sqrt(TIMES * there + 1), (m, n, here, there)
