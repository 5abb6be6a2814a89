"""The embedding gradient's long sums (-m gpu)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import paper_1806_11248_amd as g
    c = g.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("places,rows,width", [(1 << 28, 2, 256), (1 << 24, 40, 512), (5_000_000, 1, 256), (3_000_001, 33, 8)])
def test_equal_gradients_of_one_row(ctx, places, rows, width):
    """Places of the same gradient, whose additions are all rounded the same way as long as the sum's exponent stays: the worst order of a sum.  At most 512 of them are added up
    behind one another, then 512 such sums by a wave (sums of 64 and pieces of 64 of those, where ids are sorted, the rest in 64 bits), and those of 1024 waves by
    shares: fewer than 1500 roundings in all."""
    ids = torch.full((places,), rows - 1, dtype=torch.int32, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        row = torch.linspace(0.1, 2.0, width).to(dtype)
        got = ctx.embedding_backward(row.cuda().expand(places, width), ids, rows).cpu().double()
        want = row.double() * places
        assert bool(((got[rows - 1] - want).abs() <= 1500 * 2.0 ** -24 * want).all()), float(((got[rows - 1] - want).abs() / want).max())
        assert bool((got[:rows - 1] == 0).all())
        # half of them elsewhere, and added to what is there
        ids[: places // 2] = 0
        out = torch.ones(rows, width, device="cuda")
        ctx.embedding_backward(row.cuda().expand(places, width), ids, out=out, accumulate=True)
        want = row.double() * (places - places // 2 if rows > 1 else places) + 1
        assert bool(((out[rows - 1].cpu().double() - want).abs() <= 1500 * 2.0 ** -24 * want).all())
        ids.fill_(rows - 1)
