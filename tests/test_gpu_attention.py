"""Attention over ragged rows with a bias by buckets of distance, and its backward pass, against the formulas in 64 bits (-m gpu)."""
import math

import numpy as np
import pytest
import torch

from attention_ref import Reference, close, rows_of

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    import paper_1806_11248_amd as g
    c = g.Context(0)
    yield c
    c.close()


def _make(nq, nk, H, K, D, dtype, *, causal, buckets=0, far=40, room=0, fused=False, seed=0, spread=1.0, poison=True):
    """Inputs on the GPU and what the call takes.  Rows that belong to no sequence hold NaN."""
    import paper_1806_11248_amd as g
    rng = torch.Generator().manual_seed(seed)
    q_ptr = rows_of(nq)
    k_ptr = rows_of([n + room for n in nk])
    same = fused and nq == nk and room == 0
    if same:
        qkv = (torch.randn(q_ptr[-1], H + 2 * K, D, generator=rng) * spread).to(dtype).cuda()
        q, k, v = qkv.split([H, K, K], dim=1)
    else:
        q, k, v = ((torch.randn(n, h, D, generator=rng) * spread).to(dtype) for n, h in ((q_ptr[-1], H), (k_ptr[-1], K), (k_ptr[-1], K)))
        if room and poison:
            for s, n in enumerate(nk):
                k[k_ptr[s] + n:k_ptr[s + 1]] = math.nan
                v[k_ptr[s] + n:k_ptr[s + 1]] = math.inf
        q, k, v = q.cuda(), k.cuda(), v.cuda()
    cuts = g.distance_cuts(buckets, far, causal) if buckets else None
    bias = torch.randn(buckets, H, generator=rng).cuda() if buckets else None
    dout = torch.randn(q_ptr[-1], H, D, generator=rng).to(dtype).cuda()
    args = dict(q_ptr=torch.tensor(q_ptr).cuda(), k_ptr=torch.tensor(k_ptr).cuda(), max_q=max(nq), max_k=max(nk), causal=causal, bias=bias, cuts=cuts)
    if room:
        args["k_len"] = torch.tensor(nk, dtype=torch.int32).cuda()
    spans = list(zip(q_ptr[:-1], nq, k_ptr[:-1], nk))
    return q, k, v, dout, args, spans


def _reference(q, k, v, args, spans, dout=None, scale=None):
    D = q.shape[2]
    return Reference(q.cpu(), k.cpu(), v.cpu(), spans, args["causal"], D ** -0.5 if scale is None else scale,
                     None if args["bias"] is None else args["bias"].cpu(), args["cuts"], None if dout is None else dout.cpu())


def _check(ctx, made, backward=True):
    q, k, v, dout, args, spans = made
    ref = _reference(q, k, v, args, spans, dout if backward else None)
    out = ctx.attention(q, k, v, **args)
    close(out, ref.out, ref.out_tol, "out")
    saved_out, saved = ctx.attention(q, k, v, save=True, **args)
    close(saved_out, ref.out, ref.out_tol, "out of a saved pass")
    close(saved[0], ref.lse, ref.lse_tol, "lse")
    if not backward:
        return
    grads = ctx.attention_backward(dout, q, k, v, saved_out, saved, **args)
    again = ctx.attention_backward(dout, q, k, v, saved_out, saved, **args)
    for name, a, b in zip(("dq", "dk", "dv", "dbias"), grads, again):
        if a is None:
            assert name == "dbias" and args["bias"] is None
            continue
        assert torch.equal(a, b), f"{name} differs from run to run"
        close(a, getattr(ref, name), getattr(ref, name + "_tol"), name)
    # rows of no sequence get zeros
    assert not grads[1].cpu()[~ref.covered_k].any() and not grads[2].cpu()[~ref.covered_k].any()


SHAPES = [
    # one token; the tile edges of 32, 64 and 128 rows; nothing at all; the last of each kind without neighbours
    ([1], [1], 1, 1, 8), ([31, 32, 33], [31, 32, 33], 2, 1, 32), ([63, 64, 65, 0, 1], [63, 64, 65, 0, 1], 4, 4, 64),
    ([127, 129, 2], [127, 129, 2], 2, 2, 128), ([257], [257], 3, 1, 96), ([40], [40], 6, 2, 80), ([70, 5], [70, 5], 2, 1, 24),
    ([50, 50], [50, 50], 2, 2, 104), ([192], [192], 1, 1, 40),
    # more keys than queries, fewer (causal: the first rows see none), none, and no queries
    ([33, 64, 100], [90, 300, 101], 4, 2, 64), ([100, 150, 40], [30, 140, 1], 2, 1, 64), ([36, 0, 50], [0, 17, 200], 2, 2, 32),
]


@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_against_the_formulas(ctx, shape, causal, dtype):
    nq, nk, H, K, D = SHAPES[shape]
    buckets = [0, 1, 2, 7, 32, 128][(shape + causal) % 6]
    _check(ctx, _make(nq, nk, H, K, D, dtype, causal=causal, buckets=buckets, far=max(60, 2 * buckets), seed=shape, fused=shape % 2 == 1))


@pytest.mark.parametrize("far,buckets", [(20, 32), (64, 33), (700, 24), (5000, 40), (100_000, 5)])
@pytest.mark.parametrize("causal", [False, True])
def test_buckets_near_and_far(ctx, far, buckets, causal):
    """Buckets of one distance, wider than a tile, wider than the rows: every way a tile's distances fall into them."""
    _check(ctx, _make([700, 321], [700, 321], 2, 1, 32, BF, causal=causal, buckets=buckets, far=far, seed=far))


def test_cuts_anywhere(ctx):
    """Cuts are the caller's: far from zero, on one side only, or none that any pair reaches."""
    for cuts in ([5, 6, 90], [-400, -399, -130], [10 ** 9], [-2 ** 31, 0, 2 ** 31 - 2]):
        made = _make([150, 40], [260, 40], 2, 2, 64, BF, causal=False, buckets=len(cuts) + 1, seed=7)
        made[4]["cuts"] = cuts
        _check(ctx, made)


# (queries, keys, heads, kv_heads, head_dim, room)
STORES = [
    ([1], [1], 1, 1, 64, 0), ([1, 1, 1], [5, 64, 333], 8, 2, 64, 7), ([1, 1], [4097, 1500], 16, 4, 128, 16), ([1] * 5, [1, 0, 2, 127, 129], 4, 4, 32, 3),
    ([2, 1, 3], [900, 3, 2500], 8, 8, 96, 1), ([4, 1], [40, 600], 6, 2, 80, 5), ([7], [3000], 4, 1, 40, 0), ([5, 0, 6], [2, 30, 6], 3, 1, 64, 2),
    ([32, 9], [333, 2000], 1, 1, 64, 0), ([1], [20_000], 32, 1, 128, 0),
]


@pytest.mark.parametrize("store", range(len(STORES)))
@pytest.mark.parametrize("causal", [False, True])
def test_new_events_against_a_store(ctx, store, causal):
    """Few query rows: the form that is split over the keys and joined; slots' unused rows hold NaN and infinities."""
    nq, nk, H, K, D, room = STORES[store]
    dtype = BF if store % 2 else HF
    made = _make(nq, nk, H, K, D, dtype, causal=causal, buckets=[0, 16, 40][store % 3], far=1000, room=room, seed=store)
    _check(ctx, made, backward=max(nk) < 5000)


def test_one_new_event_is_the_last_row_of_the_whole(ctx):
    q, k, v, dout, args, spans = _make([300], [300], 4, 2, 64, BF, causal=True, buckets=20, seed=1)
    whole = ctx.attention(q, k, v, causal=True, bias=args["bias"], cuts=args["cuts"])
    one = ctx.attention(q[-1:].contiguous(), k, v, causal=True, bias=args["bias"], cuts=args["cuts"])
    ref = _reference(q, k, v, args, spans)
    close(one, ref.out[-1:], ref.out_tol[-1:], "new event")
    close(whole[-1:], ref.out[-1:], ref.out_tol[-1:], "last row")


@pytest.mark.parametrize("dtype", [BF, HF])
def test_large_scores(ctx, dtype):
    """Scores in the hundreds, both signs: probabilities that underflow, rows that one key owns."""
    _check(ctx, _make([130, 5], [130, 5], 2, 2, 64, dtype, causal=True, buckets=8, spread=6.0, seed=2))
    q, k, v, dout, args, spans = _make([70], [70], 1, 1, 32, dtype, causal=False, buckets=4, seed=3)
    args["bias"][:] = torch.tensor([[-300.0], [80.0], [-3e38], [0.0]]).cuda()        # a bias of the type's lowest values shuts a bucket out
    ref = _reference(q, k, v, args, spans)
    out = ctx.attention(q, k, v, **args)
    close(out, ref.out, ref.out_tol, "out")


def test_minus_infinity_in_the_bias_shuts_a_bucket_out(ctx):
    """A bucket at -inf takes no part; a row all of whose keys are shut out is a row without keys."""
    made = _make([90], [90], 2, 1, 64, BF, causal=False, buckets=5, seed=4)
    q, k, v, dout, args, spans = made
    args["cuts"] = [-30, -3, 3, 30]
    args["bias"][0] = args["bias"][3] = -math.inf
    _check(ctx, made)
    args["bias"][2] = -math.inf                # the nearest too: rows at the ends keep one side, the middle both
    _check(ctx, made)
    args["bias"][:] = -math.inf
    out, saved = ctx.attention(q, k, v, save=True, **args)
    assert not out.any() and torch.isinf(saved[0]).all()
    grads = ctx.attention_backward(dout, q, k, v, out, saved, **args)
    assert all(not x.any() for x in grads)
    args["bias"][0] = 1.0                      # the first rows see nothing still
    _check(ctx, made)


def test_non_finite_values_stay_in_their_sequence(ctx):
    nq = [40, 65, 30]
    q, k, v, dout, args, spans = _make(nq, nq, 2, 1, 64, BF, causal=True, buckets=6, seed=5)
    ref = _reference(q, k, v, args, spans, dout)
    k[50], v[60], q[70], dout[80] = math.nan, math.inf, math.nan, math.nan           # all of the second sequence
    out, saved = ctx.attention(q, k, v, save=True, **args)
    dq, dk, dv, _ = ctx.attention_backward(dout, q, k, v, out, saved, **args)
    for a, b in ((0, 40), (105, 135)):
        for name, x in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv)):
            close(x[a:b], getattr(ref, name)[a:b], getattr(ref, name + "_tol")[a:b], name)
    assert torch.isnan(out[40:105]).any()


def test_gradients_against_differences(ctx):
    """Directional differences of the 64-bit values, within what the bounds of the gradients allow along the direction."""
    made = _make([60, 100], [60, 100], 4, 2, 32, HF, causal=True, buckets=9, seed=6)
    q, k, v, dout, args, spans = made
    ref = _reference(q, k, v, args, spans, dout)
    out, saved = ctx.attention(q, k, v, save=True, **args)
    grads = dict(zip(("q", "k", "v", "bias"), ctx.attention_backward(dout, q, k, v, out, saved, **args)))
    base = dict(q=q.cpu().double(), k=k.cpu().double(), v=v.cpu().double(), bias=args["bias"].cpu().double())
    g = dout.cpu().double()
    rng = torch.Generator().manual_seed(9)

    def value(x):
        return float((Reference(x["q"], x["k"], x["v"], spans, True, 32 ** -0.5, x["bias"], args["cuts"]).out * g).sum())

    for name in base:
        d = torch.randn(base[name].shape, generator=rng, dtype=torch.float64)
        h = 1e-5
        diff = (value({**base, name: base[name] + h * d}) - value({**base, name: base[name] - h * d})) / (2 * h)
        tol = float((getattr(ref, "d" + name + "_tol") * d.abs()).sum()) + 1e-6 * abs(diff) + 1e-6
        assert abs(float((grads[name].cpu().double() * d).sum()) - diff) <= tol, name


def test_rows_far_apart(ctx):
    """Strides of a fused projection with other parts between, outputs into the caller's tensor, sequences of equal length without pointers."""
    rng = torch.Generator().manual_seed(11)
    big = torch.randn(96, 3, 12, 64, generator=rng).to(BF).cuda()
    q, k, v = big[:, 0, :8], big[:, 1, 2:6], big[:, 2, 8:12]
    spans = [(0, 32, 0, 32), (32, 32, 32, 32), (64, 32, 64, 32)]
    ref = Reference(q.cpu(), k.cpu(), v.cpu(), spans, False, 64 ** -0.5)
    ptr = torch.tensor([0, 32, 64, 96]).cuda()
    wide = torch.full((96, 2, 8, 64), 7.0, dtype=BF).cuda()
    out = ctx.attention(q, k, v, q_ptr=ptr, k_ptr=ptr, max_q=32, max_k=32, out=wide[:, 1])
    assert out.data_ptr() == wide[:, 1].data_ptr() and bool((wide[:, 0] == 7.0).all())
    close(out, ref.out, ref.out_tol, "out")
    plain = ctx.attention(q[:32], k[:32], v[:32])
    assert torch.equal(plain, out[:32])


def test_pointers_beyond_the_rows_describe_nothing(ctx):
    """Row pointers come from the device unchecked: what does not lie inside the tensors is not read, and its rows are those of no sequence."""
    q, k, v, dout, args, spans = _make([40, 40], [40, 40], 2, 2, 64, BF, causal=True, buckets=4, seed=12)
    out = torch.full_like(q, 5.0)
    for bad in ([0, 10 ** 12, 80], [-5, 40, 10 ** 15], [60, 20, 10]):
        a = dict(args, q_ptr=torch.tensor(bad).cuda(), k_ptr=torch.tensor(bad).cuda())
        out.fill_(5.0)
        ctx.attention(q, k, v, out=out, **a)
        torch.cuda.synchronize()
        assert not out.any()


def test_another_stream_than_the_current_one(ctx):
    import paper_1806_11248_amd as g
    side = torch.cuda.Stream()
    other = g.Context(0, stream=side)
    try:
        q, k, v, dout, args, spans = _make([200, 77], [200, 77], 4, 2, 64, BF, causal=True, buckets=12, seed=13)
        want_out, saved = ctx.attention(q, k, v, save=True, **args)
        want = ctx.attention_backward(dout, q, k, v, want_out, saved, **args)
        side.wait_stream(torch.cuda.current_stream())
        out, saved = other.attention(q, k, v, save=True, **args)
        got = other.attention_backward(dout, q, k, v, out, saved, **args)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want_out) and all(torch.equal(a, b) for a, b in zip(got, want))
    finally:
        other.close()


def test_in_a_graph(ctx):
    """The calls allocate nothing and wait for nothing, so they can be recorded; every replay gives the eager result."""
    import paper_1806_11248_amd as g
    side = torch.cuda.Stream()
    own = g.Context(0, stream=side)
    try:
        for nq, nk in (([150, 90], [150, 90]), ([1, 1], [3000, 40])):
            q, k, v, dout, args, spans = _make(nq, nk, 4, 2, 64, BF, causal=True, buckets=12, seed=14)
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                out, saved = own.attention(q, k, v, save=True, **args)
                own.attention_backward(dout, q, k, v, out, saved, **args)
                side.synchronize()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    out, saved = own.attention(q, k, v, save=True, **args)
                    grads = own.attention_backward(dout, q, k, v, out, saved, **args)
                for step in range(3):
                    q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(step)).to(BF))
                    graph.replay()
                    side.synchronize()
                    eager, s2 = own.attention(q, k, v, save=True, **args)
                    want = own.attention_backward(dout, q, k, v, eager, s2, **args)
                    side.synchronize()
                    assert torch.equal(out, eager) and all(torch.equal(a, b) for a, b in zip(grads, want))
    finally:
        own.close()


def test_no_rows_at_all(ctx):
    q = torch.empty(0, 4, 64, dtype=BF, device="cuda")
    k = torch.empty(0, 2, 64, dtype=BF, device="cuda")
    bias = torch.ones(3, 4, device="cuda")
    ptr = torch.zeros(1, dtype=torch.int64, device="cuda")
    out, saved = ctx.attention(q, k, k, q_ptr=ptr, k_ptr=ptr, max_q=0, max_k=0, bias=bias, cuts=[-1, 0], save=True)
    dq, dk, dv, dbias = ctx.attention_backward(q, q, k, k, out, saved, q_ptr=ptr, k_ptr=ptr, max_q=0, max_k=0, bias=bias, cuts=[-1, 0])
    assert out.shape == q.shape and not dbias.any()


def test_refusals(ctx):
    import ctypes as C
    import paper_1806_11248_amd as g
    b = g.binding
    q, k, v, dout, args, spans = _make([20], [20], 4, 2, 64, BF, causal=True, buckets=4, seed=15)
    out, saved = ctx.attention(q, k, v, save=True, **args)

    def refused(code, call):
        with pytest.raises(g.GbtError) as e:
            call()
        assert e.value.code == code

    with pytest.raises(TypeError):
        ctx.attention(q, k.half(), v, **args)
    with pytest.raises(TypeError):
        ctx.attention(q.cpu(), k, v, **args)
    with pytest.raises(TypeError):
        ctx.attention(q, k, v[:, :1], **args)
    with pytest.raises(TypeError):
        ctx.attention(q, k, v, **dict(args, cuts=[1]))
    with pytest.raises(TypeError):
        ctx.attention(q, k, v, **dict(args, bias=args["bias"][:, :2]))
    with pytest.raises(TypeError):
        ctx.attention(q, k, v, **dict(args, q_ptr=args["q_ptr"].int()))
    with pytest.raises(TypeError):
        ctx.attention(q, k, v, **dict(args, k_len=torch.ones(3, dtype=torch.int32, device="cuda")))
    with pytest.raises(TypeError):
        ctx.attention_backward(dout[:5], q, k, v, out, saved, **args)
    with pytest.raises(TypeError):
        ctx.attention_backward(dout, q, k, v, out, (saved[0][:, :3], saved[1]), **args)
    refused(b.EUNSUPPORTED, lambda: ctx.attention(q.float(), k.float(), v.float(), **args))
    odd = torch.zeros(20, 2, 12, dtype=BF, device="cuda")
    refused(b.EUNSUPPORTED, lambda: ctx.attention(odd, odd, odd))
    wide = torch.zeros(20, 2, 136, dtype=BF, device="cuda")
    refused(b.EUNSUPPORTED, lambda: ctx.attention(wide, wide, wide))
    three = torch.zeros(20, 3, 64, dtype=BF, device="cuda")
    refused(b.EINVAL, lambda: ctx.attention(q, three, three))
    refused(b.EINVAL, lambda: ctx.attention(q, k, v, **dict(args, cuts=[1, 1, 2])))
    refused(b.EINVAL, lambda: ctx.attention(q, k, v, **dict(args, scale=math.inf)))
    for wrong in (torch.empty_like(q[:1]).expand(20, 4, 64), torch.empty_like(q[:, :1]).expand(20, 4, 64),
                  torch.empty(64 * 30, dtype=BF, device="cuda").as_strided((20, 4, 64), (64, 64, 1)),
                  torch.empty(64 * 90, dtype=BF, device="cuda").as_strided((20, 4, 64), (256, 56, 1))):
        refused(b.EINVAL, lambda: ctx.attention(q, k, v, out=wrong, **args))
    by_head = torch.empty(4, 20, 64, dtype=BF, device="cuda").transpose(0, 1)
    assert torch.equal(ctx.attention(q, k, v, out=by_head, **args), out)
    refused(b.EINVAL, lambda: ctx.attention(q, k, v, **dict(args, max_q=1 << 29)))          # more workgroups than a launch can have
    refused(b.EINVAL, lambda: ctx.attention(q, k, v, **dict(args, max_k=(1 << 29) + 1)))
    shifted = torch.zeros(20 * 4 * 64 + 8, dtype=BF, device="cuda")[4:20 * 4 * 64 + 4].view(20, 4, 64)
    refused(b.EINVAL, lambda: ctx.attention(shifted, k, v, **args))
    many = torch.zeros(300, 4, device="cuda")
    refused(b.EUNSUPPORTED, lambda: ctx.attention(q, k, v, **dict(args, bias=many, cuts=list(range(299)))))
    # the C entry: missing arguments and short workspaces come back as codes, nothing is written
    lib, n = ctx.lib, None
    assert lib.gbt_attention(None, n, n, n, n, n, n, n, n, 0) == b.EINVAL
    assert lib.gbt_attention(ctx.h, n, n, n, n, n, n, n, n, 0) == b.EINVAL
    p, keep = ctx._attention_params(q, k, args["q_ptr"], args["k_ptr"], None, 20, 20, True, None, args["bias"], args["cuts"])
    views = [C.byref(b._heads(t, "t", BF)) for t in (dout, q, k, v, out, q, k, v)]
    need = lib.gbt_attention_backward_workspace_bytes(C.byref(p))
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    dbias = torch.full((4, 4), 3.0, device="cuda")
    tail = [*views[5:], b._ptr(dbias), b._ptr(ws)]
    assert lib.gbt_attention_backward(ctx.h, C.byref(p), *views[:5], b._ptr(saved[0]), n, *tail, need - 1) == b.ENOMEM
    assert lib.gbt_attention_backward(ctx.h, C.byref(p), *views[:5], n, n, *tail, need) == b.EINVAL
    p.max_q = -1
    assert lib.gbt_attention_backward_workspace_bytes(C.byref(p)) == 0
    assert lib.gbt_attention_backward(ctx.h, C.byref(p), *views[:5], b._ptr(saved[0]), n, *tail, need) == b.EINVAL
    torch.cuda.synchronize()
    assert bool((dbias == 3.0).all())



def test_without_what_rounding_took(ctx):
    """saved without its second part: dk, dv and dbias as exact as ever, dq within the bounds of a delta of the rounded out."""
    made = _make([80], [80], 2, 2, 64, BF, causal=False, buckets=5, seed=16)
    q, k, v, dout, args, spans = made
    ref = _reference(q, k, v, args, spans, dout)
    out, saved = ctx.attention(q, k, v, save=True, **args)
    dq, dk, dv, dbias = ctx.attention_backward(dout, q, k, v, out, (saved[0], None), **args)
    for name, x in (("dk", dk), ("dv", dv), ("dbias", dbias)):
        close(x, getattr(ref, name), getattr(ref, name + "_tol"), name)
    assert float((dq.cpu().double() - ref.dq).norm() / ref.dq.norm()) < 2.0 ** -7


def test_offsets_beyond_32_bits(ctx):
    """Rows whose bytes lie beyond 4 GB: at the end of a long store, and far apart."""
    H, D = 8, 128
    rows = (1 << 32) // (2 * H * D) + 5_000
    k, v = (torch.zeros(rows, H, D, dtype=BF, device="cuda") for _ in range(2))
    n = [700, 1, 300]
    ptr = [rows - 2_000, rows - 1_200, rows - 900, rows - 600]
    rng = torch.Generator().manual_seed(20)
    small = [torch.randn(2_000, H, D, generator=rng).to(BF) for _ in range(2)]
    for big, x in ((k, small[0]), (v, small[1])):
        big[-2_000:] = x.cuda()
    for m in (1, 150):                     # new events, and blocks of queries with their gradients
        q = torch.randn(3 * m, H, D, generator=rng).to(BF).cuda()
        dout = torch.randn(3 * m, H, D, generator=rng).to(BF).cuda()
        args = dict(q_ptr=torch.arange(4, device="cuda") * m, k_ptr=torch.tensor(ptr, device="cuda"), k_len=torch.tensor(n, dtype=torch.int32, device="cuda"),
                    max_q=m, max_k=700)
        spans = [(i * m, m, ptr[i] - (rows - 2_000), n[i]) for i in range(3)]
        ref = Reference(q.cpu(), *small, spans, False, D ** -0.5, None, None, dout.cpu())
        out, saved = ctx.attention(q, k, v, save=True, **args)
        close(out, ref.out, ref.out_tol, "out")
        if m > 1:
            dq, dk, dv, _ = ctx.attention_backward(dout, q, k, v, out, saved, **args)
            close(dq, ref.dq, ref.dq_tol, "dq")
            close(dk[-2_000:], ref.dk, ref.dk_tol, "dk")
            close(dv[-2_000:], ref.dv, ref.dv_tol, "dv")
            assert not dk[:-2_000].any()
            del dk, dv
    del k, v
    # 300 rows of 2^23 elements each, of which a head is used: 5 GB
    wide = torch.zeros(300, 1 << 23, dtype=BF, device="cuda")
    x = torch.randn(300, 3, 64, generator=rng).to(BF)
    wide[:, :192] = x.view(300, 192).cuda()
    q, k, v = (wide[:, 64 * i:64 * i + 64].unflatten(1, (1, 64)) for i in range(3))
    ref = Reference(x[:, :1], x[:, 1:2], x[:, 2:], [(0, 300, 0, 300)], True, 64 ** -0.5)
    close(ctx.attention(q, k, v, causal=True), ref.out, ref.out_tol, "out")
    close(ctx.attention(q[-3:], k, v, causal=True), ref.out[-3:], ref.out_tol[-3:], "out")


def test_a_full_table_of_buckets_against_a_store(ctx):
    """128 buckets and 32 columns of 128 elements: the most LDS that the form for few rows takes."""
    _check(ctx, _make([1, 1], [700, 90], 32, 1, 128, BF, causal=True, buckets=128, far=600, room=4, seed=21), backward=False)


def test_parts_of_a_block_of_keys(ctx):
    """Few blocks of keys for many query heads and long queries: a block's workgroups, by heads and by queries, and the sum of their parts."""
    for nq, nk, H, K, D in (([1500], [90], 6, 1, 64), ([900, 10], [130, 260], 4, 2, 128), ([600], [600], 5, 1, 96), ([2100], [40], 1, 1, 32)):
        _check(ctx, _make(nq, nk, H, K, D, BF, causal=False, buckets=12, seed=22))
        _check(ctx, _make(nq, nk, H, K, D, HF, causal=True, buckets=12, seed=23))


def test_many_sequences(ctx):
    """More (sequence, head) units than XCDs, in numbers that no eighth divides; most sequences empty or short."""
    rng = np.random.default_rng(24)
    nq = [int(x) for x in rng.integers(0, 40, 90)]
    nq[13] = 300
    _check(ctx, _make(nq, nq, 3, 1, 16, BF, causal=True, buckets=6, seed=25))
    _check(ctx, _make(nq[:20], nq[:20], 3, 3, 16, HF, causal=False, buckets=6, seed=26))


def test_rows_of_no_sequence_get_zeros(ctx):
    """Before the first sequence, behind the last, beyond k_len and beyond the longest: whatever memory held, and whatever q, k and v hold there."""
    rng = torch.Generator().manual_seed(30)
    H, K, D = 4, 2, 64
    for nq, nk, room, causal in (([150, 0, 90], [150, 20, 90], 0, True), ([30, 400, 2], [260, 400, 1], 9, False), ([1, 2, 0], [300, 1500, 4], 70, True), ([0, 0], [5, 0], 3, False)):
        q_ptr, k_ptr = [7 + x for x in rows_of(nq)], [5 + x for x in rows_of([n + room for n in nk])]
        q, dout = (torch.randn(q_ptr[-1] + 1_000, H, D, generator=rng).to(BF) for _ in range(2))
        k, v = (torch.randn(k_ptr[-1] + 300, K, D, generator=rng).to(BF) for _ in range(2))
        spans = list(zip(q_ptr[:-1], nq, k_ptr[:-1], nk))
        bias, cuts = torch.randn(5, H, generator=rng), [-90, -7, 0, 12]
        ref = Reference(q, k, v, spans, causal, D ** -0.5, bias, cuts, dout)
        for t, covered in ((q, ref.covered_q), (dout, ref.covered_q), (k, ref.covered_k), (v, ref.covered_k)):
            t[~covered] = math.nan
        q, k, v, dout = q.cuda(), k.cuda(), v.cuda(), dout.cuda()
        args = dict(q_ptr=torch.tensor(q_ptr).cuda(), k_ptr=torch.tensor(k_ptr).cuda(), k_len=torch.tensor(nk, dtype=torch.int32).cuda() if room else None,
                    max_q=max(nq), max_k=max(nk), causal=causal, bias=bias.cuda(), cuts=cuts)
        for _ in range(3):                 # memory that held something else before
            torch.full((q.numel() + 4 * k.numel(),), math.nan, dtype=BF, device="cuda")
            out, saved = ctx.attention(q, k, v, save=True, **args)
            got = (out, *ctx.attention_backward(dout, q, k, v, out, saved, **args))
        for name, x in zip(("out", "dq", "dk", "dv", "dbias"), got):
            if name != "dbias":
                covered = ref.covered_k if name in ("dk", "dv") else ref.covered_q
                assert not x.cpu()[~covered].any(), name
            close(x, getattr(ref, name), getattr(ref, name + "_tol"), name)
    # more rows than n_seq * max
    q = torch.randn(50, H, D, generator=rng).to(BF).cuda()
    none = torch.zeros(1, dtype=torch.int64, device="cuda")
    out = torch.full_like(q, 3.0)
    ctx.attention(q, q, q, q_ptr=none, k_ptr=none, max_q=0, max_k=0, out=out)
    assert not out.any()


def test_many_gaps(ctx):
    """More sequences than the lanes that look for gaps between them."""
    n, room = 20_000, 3
    rng = torch.Generator().manual_seed(31)
    k_len = torch.randint(0, 4, (n,), generator=rng, dtype=torch.int32)
    k, q, dout = (torch.randn(rows, 1, 8, generator=rng).to(BF).cuda() for rows in (n * room, n, n))
    k_ptr = (torch.arange(n + 1) * room).cuda()
    args = dict(q_ptr=torch.arange(n + 1).cuda(), k_ptr=k_ptr, k_len=k_len.cuda(), max_q=1, max_k=room)
    for _ in range(2):
        torch.full((4 * k.numel(),), math.nan, dtype=BF, device="cuda")
        out, saved = ctx.attention(q, k, k, save=True, **args)
        dq, dk, dv, _ = ctx.attention_backward(dout, q, k, k, out, saved, **args)
    unused = (torch.arange(room) >= k_len[:, None]).flatten()
    assert not dk.cpu()[unused].any() and not dv.cpu()[unused].any()
    assert not out.cpu()[k_len == 0].any() and not dq.cpu()[k_len == 0].any()
    for x in (out, dq, dk, dv):
        assert torch.isfinite(x).all()


@pytest.mark.parametrize("nq", [1, 200])
def test_low_values_in_the_bias_shut_a_bucket_out(ctx, nq):
    """Whichever low value stands for a mask, results are those of -inf; rows that it leaves without keys are zeros, with zero gradients."""
    q, k, v, dout, args, spans = _make([nq, nq], [200, 330], 4, 2, 64, BF, causal=False, buckets=4, far=40, seed=32, spread=8.0)
    bias = args["bias"]
    for shut in ([0], [1, 2], [0, 1, 2, 3]):
        want = None
        for low in (-math.inf, torch.finfo(torch.float32).min, -1e10, -1e9, -2e5):
            args["bias"] = bias.clone()
            args["bias"][shut] = low
            out, saved = ctx.attention(q, k, v, save=True, **args)
            got = (out, saved[0], *ctx.attention_backward(dout, q, k, v, out, saved, **args))
            if want is None:
                want = got
                ref = _reference(q, k, v, args, spans, dout)
                close(out, ref.out, ref.out_tol, "out")
            assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert not any(x.any() for i, x in enumerate(want) if i != 1)


def test_a_graph_keeps_its_workspace(ctx):
    """A graph recorded before a larger call: its replays write to no memory that has been given back since."""
    import paper_1806_11248_amd as g
    side = torch.cuda.Stream()
    own = g.Context(0, stream=side)
    try:
        with torch.cuda.stream(side):
            small = _make([150, 90], [150, 90], 4, 2, 64, BF, causal=True, buckets=12, seed=40)
            large = _make([700] * 6, [700] * 6, 4, 2, 64, BF, causal=True, buckets=12, seed=41)
            few, many = (_make([1, 1], [n, 40], 4, 2, 64, BF, causal=True, buckets=12, seed=n) for n in (3_000, 30_000))

            def run(made):
                q, k, v, dout, args, _ = made
                out, saved = own.attention(q, k, v, save=True, **args)
                return (out, *own.attention_backward(dout, q, k, v, out, saved, **args))
            eager = [run(m) for m in (small, few)]
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                recorded = [run(m) for m in (small, few)]
            for _ in range(2):
                run(large), run(many)                      # larger workspaces take the place of the first ones
                others = [torch.full((n,), 9, dtype=torch.uint8, device="cuda") for n in [1 << 12, 1 << 16, 1 << 18, 1 << 20, 1 << 21, 1 << 22] for _ in range(4)]
                graph.replay()
                side.synchronize()
                assert all(bool((x == 9).all()) for x in others)
                assert all(torch.equal(a, b) for x, y in zip(recorded, eager) for a, b in zip(x, y))
    finally:
        own.close()


@pytest.mark.parametrize("nq", [1, 90])
def test_broadcast_inputs(ctx, nq):
    """Heads and rows that are the same memory; gradients are those of each element, for the caller to add up."""
    rng = torch.Generator().manual_seed(50)
    q = torch.randn(nq, 1, 64, generator=rng).to(BF).expand(nq, 4, 64)
    k = torch.randn(200, 1, 64, generator=rng).to(BF).expand(200, 2, 64)
    v = torch.randn(1, 2, 64, generator=rng).to(BF).expand(200, 2, 64)
    dout = torch.randn(1, 4, 64, generator=rng).to(BF).expand(nq, 4, 64)
    ref = Reference(q, k, v, [(0, nq, 0, 200)], True, 64 ** -0.5, None, None, dout)
    base = [torch.randn(0)] * 4
    for i, x in enumerate((q, k, v, dout)):
        base[i] = x[:x.stride(0) and x.shape[0] or 1, :x.stride(1) and x.shape[1] or 1].cuda().expand(x.shape)
    q, k, v, dout = base
    assert 0 in q.stride() + k.stride() and v.stride(0) == 0 and (nq == 1 or dout.stride(0) == 0)
    out, saved = ctx.attention(q, k, v, causal=True, save=True)
    close(out, ref.out, ref.out_tol, "out")
    for name, x in zip(("dq", "dk", "dv"), ctx.attention_backward(dout, q, k, v, out, saved, causal=True)):
        close(x, getattr(ref, name), getattr(ref, name + "_tol"), name)


@pytest.mark.parametrize("seqs", [2, 31, 33, 64, 65])
@pytest.mark.parametrize("causal", [False, True])
def test_sequences_by_length(ctx, seqs, causal):
    """Lengths alike, apart, none; queries and keys of different lengths: whichever is taken first, each is taken once."""
    rng = np.random.default_rng(seqs)
    nq = [int(x) for x in rng.choice([0, 1, 127, 128, 129, 200, 300, 512], seqs)]
    nk = [int(x) for x in rng.choice([0, 1, 128, 140, 260, 512], seqs)]
    nq[0], nk[-1] = 520, 513
    _check(ctx, _make(nq, nk, 1, 1, 8, BF, causal=causal, buckets=5, seed=seqs))
    _check(ctx, _make(nq[:5], nk[-5:], 2, 1, 128, HF, causal=causal, buckets=5, seed=seqs, room=9))


def test_causal_sequences_by_length(ctx):
    """Causal histories beyond what the L2 holds are taken by length too; most of the rows belong to one that is not looked at."""
    rows, H, D = 140_000, 1, 128                       # 4 * 140,000 * 128 bytes of keys and values
    nq, nk = [300, 10, 0, 420, 257], [300, 200, 40, 500, 257]
    q, k, v, dout, args, spans = _make(nq, nk, H, H, D, BF, causal=True, buckets=6, seed=60)
    big = {}
    for name, x in (("q", q), ("k", k), ("v", v), ("dout", dout)):
        big[name] = torch.zeros(rows, H, D, dtype=BF, device="cuda")
        big[name][:len(x)] = x
    out, saved = ctx.attention(big["q"], big["k"], big["v"], save=True, **args)
    got = ctx.attention_backward(big["dout"], big["q"], big["k"], big["v"], out, saved, **args)
    ref = _reference(q, k, v, args, spans, dout)
    for name, x, n in zip(("out", "dq", "dk", "dv"), (out, *got), (len(q), len(q), len(k), len(k))):
        close(x[:n], getattr(ref, name), getattr(ref, name + "_tol"), name)
        assert not x[n:].any()
    close(got[3], ref.dbias, ref.dbias_tol, "dbias")


@pytest.mark.parametrize("causal", [False, True])
def test_parts_of_a_block_of_keys_in_a_store(ctx, causal):
    """A block's parts, of sequences whose slots are a small share of a store's rows, and of as many rows as the longest sequences would have or fewer."""
    for nq, nk, rows, H, K, D in (([1500, 700], [90, 300], 60_000, 6, 1, 64), ([900, 10, 300], [130, 260, 0], 20_000, 4, 2, 128), ([900, 10], [130, 260], 390, 4, 2, 128)):
        q, k, v, dout, args, spans = _make(nq, nk, H, K, D, BF, causal=causal, buckets=12, seed=70)
        at = [rows - sum(nk) + x for x in rows_of(nk)]
        ref = _reference(q, k, v, args, spans, dout)
        big_k, big_v = (torch.full((rows, K, D), math.nan, dtype=BF, device="cuda") for _ in range(2))
        big_k[at[0]:], big_v[at[0]:] = k, v
        args["k_ptr"] = torch.tensor(at).cuda()
        args["k_len"] = torch.tensor(nk, dtype=torch.int32).cuda()
        out, saved = ctx.attention(q, big_k, big_v, save=True, **args)
        dq, dk, dv, dbias = ctx.attention_backward(dout, q, big_k, big_v, out, saved, **args)
        for name, x in (("dq", dq), ("dk", dk[at[0]:]), ("dv", dv[at[0]:]), ("dbias", dbias)):
            close(x, getattr(ref, name), getattr(ref, name + "_tol"), name)
        assert not dk[:at[0]].any() and not dv[:at[0]].any()


def test_a_loose_longest_sequence_costs_idle_workgroups_and_no_more(ctx):
    """Up to 64 sequences are put in order by their lengths, by every workgroup for itself: the same launch but for one more sequence, and so
    without that order, takes as long, however far the longest sequence lies below the bound that the caller gives."""
    def call(seqs, bound):
        nq = [100 + 3 * s for s in range(seqs)]
        q, k, v, dout, args, spans = _make(nq, nq, 1, 1, 64, BF, causal=False, seed=71)
        args.update(max_q=bound, max_k=bound)
        return q, k, v, args, spans

    took = {}
    for seqs in (64, 65):
        q, k, v, args, spans = call(seqs, 1 << 20)
        out = ctx.attention(q, k, v, **args)
        ref = _reference(q, k, v, args, spans)
        close(out, ref.out, ref.out_tol, "out")
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        for _ in range(5):
            ctx.attention(q, k, v, out=out, **args)
        end.record()
        end.synchronize()
        took[seqs] = begin.elapsed_time(end) / 5
    print(took)
    assert took[64] < 3 * took[65]


def test_without_the_longest_sequences(ctx):
    """max_q and max_k left out are what the pointers say: the same results as with them, for many sequences, single events and other streams."""
    import paper_1806_11248_amd as g
    rng = np.random.default_rng(72)
    many = [int(x) for x in rng.integers(0, 40, 4_000)]
    for nq, nk, room in ((many, many, 0), ([1] * 64, [int(x) for x in rng.integers(0, 900, 64)], 5), ([300, 0, 70], [40, 7, 500], 0), ([0, 0], [3, 0], 0), ([50], [60], 0)):
        q, k, v, dout, args, spans = _make(nq, nk, 4, 2, 64, BF, causal=True, buckets=6, room=room, seed=73)
        want, saved = ctx.attention(q, k, v, save=True, **args)
        grads = ctx.attention_backward(dout, q, k, v, want, saved, **args)
        for gone in (("max_q",), ("max_k",), ("max_q", "max_k")):
            less = {n: x for n, x in args.items() if n not in gone}
            out, saved = ctx.attention(q, k, v, save=True, **less)
            assert torch.equal(out, want)
            if len(nq) > 1:
                assert all(torch.equal(a, b) for a, b in zip(ctx.attention_backward(dout, q, k, v, out, saved, **less), grads))
    # the context's own stream, and a graph, in which nothing can be read: all rows there
    side = torch.cuda.Stream()
    own = g.Context(0, stream=side)
    try:
        q, k, v, dout, args, spans = _make([90, 20, 150], [90, 20, 150], 4, 2, 64, BF, causal=True, buckets=6, seed=74)
        ref = _reference(q, k, v, args, spans)
        less = {n: x for n, x in args.items() if n not in ("max_q", "max_k")}
        side.wait_stream(torch.cuda.current_stream())
        out = own.attention(q, k, v, **less)
        side.synchronize()
        close(out, ref.out, ref.out_tol, "out")
        with torch.cuda.stream(side):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                out = own.attention(q, k, v, **less)
            for _ in range(2):
                out.zero_()
                graph.replay()
                side.synchronize()
                close(out, ref.out, ref.out_tol, "out of a graph")
    finally:
        own.close()


def _one_key_and_many_small_ones(n, nq, seed):
    """Queries that one key, the first, owns but for n others at 2^-26 of it, which are 2^-6 of the sum together where n is 2^20."""
    q = torch.full((nq, 1, 8), 1.0, dtype=HF)
    k = torch.zeros(n, 1, 8, dtype=HF)
    k[0] = 26.0 * math.log(2.0) / 8.0
    v = torch.full((n, 1, 8), -16.0, dtype=HF) + torch.randn(n, 1, 8, generator=torch.Generator().manual_seed(seed)).to(HF)
    v[0] = 1.0
    return q, k, v


@pytest.mark.parametrize("nq", [1, 40, 200])
def test_float16_keeps_small_probabilities(ctx, nq):
    """What many keys of little weight add up to is in the result: none of them is below what a product in float16 holds."""
    q, k, v = _one_key_and_many_small_ones(1 << 17, nq, 80)
    ref = Reference(q, k, v, [(0, nq, 0, len(k))], False, 1.0)
    out = ctx.attention(q.cuda(), k.cuda(), v.cuda(), scale=1.0)
    close(out, ref.out, ref.out_tol, "out")


def _off(got, want):
    """Relative errors of dq, dk and dv, and those of rounding the exact ones to float16 alone."""
    def rel(x, y):
        return float((x.cpu().double() - y).norm() / y.norm())

    return [rel(x, y) for x, y in zip(got, want)], [rel(y.to(HF), y) for y in want]


@pytest.mark.parametrize("D,causal", [(64, False), (128, True), (40, True)])
def test_float16_gradients_of_small_gradients(ctx, D, causal):
    """All gradients are linear in dout, so a smaller dout gives them as exactly, but for what the type cannot hold of them: twice each, for
    roundings that fall differently."""
    for exponent in (8, 10, 12):
        q, k, v, dout, args, spans = _make([2048], [2048], 2, 1, D, HF, causal=causal, seed=81)
        small = (dout.float() * 2.0 ** -exponent).to(HF)
        large = (small.float() * 2.0 ** exponent).to(HF)                     # dout, but for what small cannot hold
        assert torch.equal(small.double() * 2.0 ** exponent, large.double())
        ref = _reference(q, k, v, args, spans, large)
        out, saved = ctx.attention(q, k, v, save=True, **args)
        of_large, _ = _off(ctx.attention_backward(large, q, k, v, out, saved, **args)[:3], (ref.dq, ref.dk, ref.dv))
        of_small, rounding = _off(ctx.attention_backward(small, q, k, v, out, saved, **args)[:3], [x * 2.0 ** -exponent for x in (ref.dq, ref.dk, ref.dv)])
        print(exponent, of_large, of_small, rounding)
        for a, b, r in zip(of_small, of_large, rounding):
            assert a <= 2 * b + 2 * r


@pytest.mark.parametrize("nk", [40, 400])
def test_float16_scores_gradients_beyond_the_type(ctx, nk):
    """Gradients of scores above 65504, of queries and keys that are small, so that their own gradients are not."""
    q, k, v, dout, args, spans = _make([nk], [nk], 2, 1, 64, HF, causal=True, seed=82)
    q, k, v, dout = q * 2.0 ** -6, k * 2.0 ** -6, v * 256.0, dout * 2.0 ** -3
    large = dout * 2.0 ** 15
    out, saved = ctx.attention(q, k, v, save=True, **args)
    ref = _reference(q, k, v, args, spans, dout)
    of_dout, _ = _off(ctx.attention_backward(dout, q, k, v, out, saved, **args)[:3], (ref.dq, ref.dk, ref.dv))
    got = ctx.attention_backward(large, q, k, v, out, saved, **args)[:3]
    of_large, rounding = _off(got, [x * 2.0 ** 15 for x in (ref.dq, ref.dk, ref.dv)])
    print(of_dout, of_large, rounding)
    assert all(torch.isfinite(x).all() for x in got)
    for a, b, r in zip(of_large, of_dout, rounding):
        assert a <= 2 * b + 2 * r


def test_float16_gradients_of_many_keys(ctx):
    """Probabilities of 2^-19 on average: what the products with dout make of them is as exact as of few keys."""
    errors = []
    for nk in (300, 400_000):
        q, k, v, dout, args, spans = _make([64], [nk], 1, 1, 16, HF, causal=False, seed=83)
        dout = dout * 1024.0
        ref = _reference(q, k, v, args, spans, dout)
        out, saved = ctx.attention(q, k, v, save=True, **args)
        errors.append(_off(ctx.attention_backward(dout, q, k, v, out, saved, **args)[:3], (ref.dq, ref.dk, ref.dv)))
    print(errors)
    for a, b, r in zip(errors[1][0][1:], errors[0][0][1:], errors[1][1][1:]):         # dk and dv
        assert a <= 2 * b + 2 * r


@pytest.mark.parametrize("group,nq", [(1, 32), (1, 33), (1, 65), (3, 10), (3, 11), (3, 22), (4, 8), (4, 9), (4, 17), (16, 2), (16, 3), (32, 1), (33, 1)])
def test_around_what_the_form_for_few_rows_takes(ctx, group, nq):
    """32 pairs of query and head for a key head and a few more: both forms, of several pieces of the keys and of one."""
    for causal in (False, True):
        _check(ctx, _make([nq, max(1, nq - 1), 0], [5_000, 40, 9], 2 * group, 2, 64, BF, causal=causal, buckets=9, far=300, room=4, seed=90), backward=False)


@pytest.mark.parametrize("store", range(len(STORES)))
@pytest.mark.parametrize("dtype", [BF, HF])
def test_few_rows_round_their_result_alone(ctx, store, dtype):
    """Single new events have few numbers, in which the rounding of a probability would show: theirs are operands in two parts, so the bound
    is without it, but for the second part's own."""
    nq, nk, H, K, D, room = STORES[store]
    q, k, v, dout, args, spans = _make(nq, nk, H, K, D, dtype, causal=True, buckets=8, far=50, room=room, seed=100 + store)
    ref = _reference(q, k, v, args, spans)
    spread = _reference(q, k, v.abs(), args, spans).out
    u = torch.finfo(dtype).eps / 2
    close(ctx.attention(q, k, v, **args), ref.out, ref.out_tol - 1.01 * u * spread + 1.01 * u * u * spread, "out")


@pytest.mark.parametrize("D", [32, 64, 80, 128])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_few_keys_round_their_result_alone(ctx, D, dtype):
    """Calls of at most 64 keys a sequence likewise, in the form for blocks of queries: the bound is without the rounding of probabilities."""
    nq = [40, 64, 1, 300, 63, 33, 0, 128]
    nk = [40, 64, 1, 64, 2, 60, 5, 20]
    for causal in (False, True):
        q, k, v, dout, args, spans = _make(nq, nk, 4, 2, D, dtype, causal=causal, buckets=8, far=50, seed=120)
        ref = _reference(q, k, v, args, spans)
        spread = _reference(q, k, v.abs(), args, spans).out
        u = torch.finfo(dtype).eps / 2
        close(ctx.attention(q, k, v, **args), ref.out, ref.out_tol - 1.01 * u * spread + 1.01 * u * u * spread, "out")
