"""Head norms with rotation: inputs of which a wave has many rows, and what only the C entry points can be asked for (-m gpu).  Bounds: tower_ref."""
import ctypes as C

import pytest
import torch

from tower_ref import TINY, U, places, rotate

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
