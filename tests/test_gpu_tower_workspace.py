"""What the workspaces of the operators around a tower held before a call does not matter (-m gpu)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import paper_1806_11248_amd as g
    c = g.Context(0)
    yield c
    c.close()


def _check(ctx, key, call):
    want = [t.clone() for t in call()]
    for byte in (0xFF, 0x00, 0x3C):
        ctx.workspace(key, 1).fill_(byte)                                        # NaN in every type, zeros, ones and a half
        assert all(torch.equal(a, b) for a, b in zip(call(), want))


@pytest.mark.parametrize("places,rows,width", [(5_000, 700, 24), (100_003, 12, 64), (60_000, 40, 40), (40_000, 70_000, 520), (200_000, 2, 200)])
def test_embedding_gradient(ctx, places, rows, width):
    ids = (rows * torch.rand(places, generator=torch.Generator().manual_seed(1)) ** 4).long().clamp_max(rows - 1).cuda()
    ids[::50] = -1
    dout = torch.randn(places, width, generator=torch.Generator().manual_seed(2)).cuda()
    _check(ctx, "embedding", lambda: [ctx.embedding_backward(dout, ids, rows)])


@pytest.mark.parametrize("rows,heads,kv_heads,dim", [(3, 1, 1, 8), (5_000, 8, 2, 64), (700, 5, 3, 40)])
def test_head_norms_gradient(ctx, rows, heads, kv_heads, dim):
    import paper_1806_11248_amd as g
    q, k, dq, dk = (torch.randn(rows, h, dim, generator=torch.Generator().manual_seed(h)).to(torch.bfloat16).cuda() for h in (heads, kv_heads, heads, kv_heads))
    turns = g.rotation_turns(dim)
    _check(ctx, "norm_rotate", lambda: list(ctx.norm_rotate_backward(dq, dk, q, k, None, None, turns)))


def test_orthogonalised_updates(ctx):
    updates = [torch.randn(m, n, generator=torch.Generator().manual_seed(m)).to(t).cuda()
               for m, n, t in ((130, 70, torch.float32), (300, 1000, torch.bfloat16), (1000, 800, torch.float32), (7, 500, torch.float16), (40, 40, torch.float32))]
    lst = ctx.matrix_list(updates, [torch.zeros_like(u) for u in updates])
    _check(ctx, "orthogonalise", lambda: ctx.orthogonalise(lst))
