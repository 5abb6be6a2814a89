"""The operators for rows that come with a history of events, as workloads.

A table's row may have a history beside its columns: the payments of a customer, the readings of a machine.  A small attention
tower reads it, its output joins the margin of the trees, and both learn from the same gradients.  The operators:

  attend   attention over ragged histories (packed rows and row pointers, as the library's sparse rows are stored), with a learned
           bias for each bucket of distance: scoring, for whole histories and for single new events against a stored one
  train    the same and its backward pass: out, and the gradients of q, k, v and of the bias table
  clip     the global norm over many gradient tensors, and the gradients scaled down to it

A case is a dict of plain values.  For attend and train: seqs histories, whose numbers of queries lie in q_lo..q_hi and of keys in
k_lo..k_hi (k_hi = 0: as many as queries), heads query heads, kv_heads key heads, dim elements a head, buckets of distance that reach
back to `far` events, causal or not, `fused`: q, k and v are parts of one projection's output.  For clip: tensors of lo..hi elements,
a share `half` of them in 16 bits, and `over`: the norm as a multiple of the limit.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _attend(name, kind, seqs, q_lo, q_hi, heads, kv_heads, dim, dtype="bf16", k_lo=0, k_hi=0, buckets=32, far=128, causal=True,
            fused=False, lengths=0):
    return dict(name=name, kind=kind, seqs=seqs, q_lo=q_lo, q_hi=q_hi, k_lo=k_lo, k_hi=k_hi, heads=heads, kv_heads=kv_heads, dim=dim,
                dtype=dtype, buckets=buckets, far=far, causal=causal, fused=fused, lengths=lengths)


def _clip(name, tensors, lo, hi, half, over, lengths=0):
    return dict(name=name, kind="clip", tensors=tensors, lo=lo, hi=hi, half=half, over=over, lengths=lengths)


def listed():
    return [
        # the smallest call: one new event for each of four rows, scored against short stored histories
        _attend("attend_new_event", "attend", 4, 1, 1, 8, 2, 64, k_lo=150, k_hi=500),
        # the same against long histories, where the stored keys and values are what there is to read
        _attend("attend_long_store", "attend", 16, 1, 1, 16, 4, 128, k_lo=2_000, k_hi=30_000, far=4_096),
        # a few new events at a time for many rows
        _attend("attend_few_events", "attend", 64, 1, 7, 8, 8, 64, dtype="f16", k_lo=30, k_hi=3_000, buckets=24, far=300),
        # whole histories of ordinary length, read in both directions
        _attend("attend_ragged", "attend", 24, 100, 1_000, 8, 8, 64, dtype="f16", causal=False, fused=True),
        # one long history, the largest scoring call
        _attend("attend_long", "attend", 1, 8_192, 8_192, 16, 4, 128, far=2_048, buckets=40),
        # a small training batch of short histories
        _attend("train_short", "train", 32, 5, 60, 4, 4, 32, buckets=16, far=50),
        # an ordinary one
        _attend("train_ragged", "train", 16, 100, 1_000, 8, 8, 64, fused=True),
        # odd lengths, a head size that is no power of two, shared key heads, both directions
        _attend("train_odd", "train", 5, 301, 777, 6, 2, 80, dtype="f16", buckets=21, far=200, causal=False),
        # the largest training batch: long histories
        _attend("train_long", "train", 2, 4_000, 4_096, 16, 4, 128, far=1_024, buckets=40),
        # the gradients of a small tower ...
        _clip("clip_small", 14, 30, 9_000, 0.0, 3.0),
        # ... of an ordinary model: many tensors of odd sizes, some kept in 16 bits
        _clip("clip_ordinary", 150, 60, 600_000, 0.5, 2.0),
        # ... of a large one, within the limit already on most steps but not on this one
        _clip("clip_large", 220, 1_000, 5_000_000, 0.5, 1.3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "store", "train", "train", "clip"])
    seed = rng.randrange(1 << 20)
    if kind == "clip":
        hi = _log_int(rng, 1_000, 3_000_000)
        return dict(_clip("", rng.randint(1, 200), rng.randint(1, 200), hi, rng.choice([0.0, 0.5, 1.0]), rng.choice([0.5, 1.5, 4.0]), seed))
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 1, 2, 4] if kv_heads < 8 else [1, 2])
    dim = rng.choice([16, 32, 40, 64, 64, 80, 96, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    buckets = rng.randint(2, 64)
    far = _log_int(rng, 64, 4_096)
    if kind == "store":
        k_hi = _log_int(rng, 40, 20_000)
        q_hi = rng.choice([1, 1, 2, 5, 9])
        return dict(_attend("", "attend", rng.randint(1, max(1, min(40, 120_000 // k_hi))), 1, q_hi, heads, kv_heads, dim, dtype, max(q_hi, k_hi // 6), k_hi + q_hi,
                            buckets, far, True, False, seed))
    q_hi = _log_int(rng, 12, 2_500)
    seqs = max(1, min(48, _log_int(rng, 2, 48), 6_000 // q_hi))
    return dict(_attend("", kind, seqs, max(1, q_hi // 5), q_hi, heads, kv_heads, dim, dtype, 0, 0, buckets, far, rng.random() < 0.6,
                        rng.random() < 0.5, seed))


def _lengths(case):
    """The numbers of queries and keys of every history: a property of the case."""
    rng = random.Random(f"{case['lengths']} {case['seqs']} {case['q_lo']} {case['q_hi']} {case['k_lo']} {case['k_hi']}")
    nq = [rng.randint(case["q_lo"], case["q_hi"]) for _ in range(case["seqs"])]
    nk = [rng.randint(case["k_lo"], case["k_hi"]) for _ in range(case["seqs"])] if case["k_hi"] else list(nq)
    return nq, nk


def _sizes(case):
    """Elements of every gradient tensor, spread over the logarithm as a model's are, and its type."""
    rng = random.Random(f"{case['lengths']} {case['tensors']} {case['lo']} {case['hi']}")
    return [(_log_int(rng, case["lo"], case["hi"]), "bf16" if rng.random() < case["half"] else "f32") for _ in range(case["tensors"])]


def _cuts(case):
    """Ascending cuts between buckets of distance (0 = the event itself, negative = the past): one bucket for each of the nearest
    events, then buckets that grow with the distance; in both directions alike where the future counts too."""
    n = case["buckets"] - 1
    back = n if case["causal"] else (n + 1) // 2
    near = max(1, back // 2)
    steps, last = [], 0
    for i in range(back):
        at = i if i < near else near * (case["far"] / near) ** ((i - near + 1) / max(1, back - near))
        last = max(int(round(at)), last + 1) if i else 0
        steps.append(last)
    cuts = [-s for s in reversed(steps)]
    return cuts + [s + 1 for s in steps[:n - back]]


def _rng(seed, salt):
    return torch.Generator(device=DEV).manual_seed(seed * 7919 + salt)


def _ptr(counts):
    p = [0]
    for c in counts:
        p.append(p[-1] + c)
    return p


def _flat_like(tensors):
    """One flat buffer for each type, as an optimizer keeps them, and a part of it for each tensor."""
    parts, places, used = [], [], {}
    for t in tensors:
        at = used.get(t.dtype, 0)
        places.append((t.dtype, at))
        used[t.dtype] = at + (t.numel() + 15) // 16 * 16
    buffers = {d: torch.zeros(n, dtype=d, device=DEV) for d, n in sorted(used.items(), key=str)}
    for t, (d, at) in zip(tensors, places):
        parts.append(buffers[d][at:at + t.numel()])
    return list(buffers.values()), parts


def prepare(case, seed):
    r = _rng(seed, 1)
    if case["kind"] == "clip":
        # gradients of very different sizes, as the layers of a model have them
        grads, total = [], 0
        for i, (n, dtype) in enumerate(_sizes(case)):
            g = torch.randn(n, generator=r, device=DEV) * 10.0 ** -(i % 5)
            grads.append(g.to(TYPES[dtype]))
            total += n * 100.0 ** -(i % 5)
        flats, outs = _flat_like(grads)
        state = dict(case=case, grads=grads, outs=outs, flats=flats, max_norm=math.sqrt(total) / case["over"])
        if own:
            ctx = _context()
            state.update(ctx=ctx, plan=ctx.gradient_list(grads, outs))
        return state
    nq, nk = _lengths(case)
    H, K, D, dt = case["heads"], case["kv_heads"], case["dim"], TYPES[case["dtype"]]

    def normal(rows, heads):
        return torch.randn(rows, heads, D, generator=r, device=DEV).to(dt)

    tq, tk = sum(nq), sum(nk)
    q_ptr = _ptr(nq)
    if case["k_hi"]:
        # a store with room for every history to grow: the slots' starts, and how much of each is used
        room = [n + n // 8 + 16 for n in nk]
        k_ptr, k_len = _ptr(room), nk
        q, k, v = normal(tq, H), normal(sum(room), K), normal(sum(room), K)
    elif case["fused"]:
        k_ptr, k_len = q_ptr, None
        q, k, v = normal(tq, H + 2 * K).split([H, K, K], dim=1)
    else:
        k_ptr, k_len = q_ptr, None
        q, k, v = normal(tq, H), normal(tk, K), normal(tk, K)
    state = dict(case=case, q=q, k=k, v=v, nq=nq, nk=nk, q_ptr=q_ptr, k_ptr=k_ptr, cuts=_cuts(case), scale=1.0 / math.sqrt(D),
                 bias=torch.randn(case["buckets"], H, generator=r, device=DEV))
    if case["kind"] == "train":
        state["dout"] = normal(tq, H)
    if own:
        state["ctx"] = _context()
        state["rows"] = dict(q_ptr=torch.tensor(q_ptr, device=DEV), k_ptr=torch.tensor(k_ptr, device=DEV),
                             k_len=None if k_len is None else torch.tensor(k_len, dtype=torch.int32, device=DEV),
                             max_q=max(nq), max_k=max(nk))
    return state


_ctx = None


def _context():
    """The program's one context, on the stream that it works on."""
    global _ctx
    if _ctx is None:
        import paper_1806_11248_amd as g
        _ctx = g.Context(0)
    return _ctx


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    ctx, kind = state["ctx"], state["case"]["kind"]
    if kind == "clip":
        norm = ctx.clip_gradients(state["plan"], state["max_norm"])
        return [norm, *state["flats"]]
    args = dict(state["rows"], causal=state["case"]["causal"], scale=state["scale"], bias=state["bias"], cuts=state["cuts"])
    if kind == "attend":
        return ctx.attention(state["q"], state["k"], state["v"], **args)
    out, saved = ctx.attention(state["q"], state["k"], state["v"], save=True, **args)
    return (out, *ctx.attention_backward(state["dout"], state["q"], state["k"], state["v"], out, saved, **args))


def _chunks(state):
    """(rows of queries, rows of keys, key heads) of pieces whose score matrices are at most 2 GB."""
    group = state["case"]["heads"] // state["case"]["kv_heads"]
    for s, (nq, nk) in enumerate(zip(state["nq"], state["nk"])):
        step = max(1, (1 << 29) // max(1, group * nq * nk))
        for c0 in range(0, state["case"]["kv_heads"], step):
            yield (slice(state["q_ptr"][s], state["q_ptr"][s] + nq), slice(state["k_ptr"][s], state["k_ptr"][s] + nk),
                   slice(c0, min(c0 + step, state["case"]["kv_heads"])))


def _heads_first(x, rows, heads):
    return x[rows, heads].float().transpose(0, 1).contiguous()


def _run_plain(state):
    kind = state["case"]["kind"]
    if kind == "clip":
        return _plain_clip(state)
    H, K = state["case"]["heads"], state["case"]["kv_heads"]
    G = H // K
    causal, scale = state["case"]["causal"], state["scale"]
    cuts = torch.tensor(state["cuts"], device=DEV)
    q, k, v, bias = state["q"], state["k"], state["v"], state["bias"]
    out = torch.zeros_like(q, memory_format=torch.contiguous_format)
    if kind == "train":
        dq, dk, dv = (torch.zeros_like(x, memory_format=torch.contiguous_format) for x in (q, k, v))
        dbias = torch.zeros_like(bias)
    for rq, rk, c in _chunks(state):
        nq, nk, nc = rq.stop - rq.start, rk.stop - rk.start, c.stop - c.start
        hs = slice(c.start * G, c.stop * G)
        qs = _heads_first(q, rq, hs).view(nc, G * nq, -1)
        ks, vs = _heads_first(k, rk, c), _heads_first(v, rk, c)
        t = torch.arange(nk, device=DEV)[None, :] - (torch.arange(nq, device=DEV)[:, None] + (nk - nq))
        bucket = (cuts[:, None, None] <= t).sum(0) if t.numel() * len(cuts) < 1 << 28 else sum((x <= t).int() for x in cuts)
        s = (torch.matmul(qs, ks.transpose(1, 2).contiguous()) * scale).view(nc * G, nq, nk)
        for h in range(nc * G):
            s[h] += bias[:, c.start * G + h][bucket]
        if causal:
            s = s.masked_fill(t > 0, -math.inf)
        top = s.amax(2, keepdim=True)
        e = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
        p = e / e.sum(2, keepdim=True).clamp_min(1e-30)
        del s, e
        o = torch.matmul(p.view(nc, G * nq, nk), vs).view(nc * G, nq, -1)
        out[rq, hs] = o.transpose(0, 1).to(q.dtype)
        if kind == "attend":
            continue
        do = _heads_first(state["dout"], rq, hs).view(nc, G * nq, -1)
        pt = p.view(nc, G * nq, nk).transpose(1, 2).contiguous()
        dv[rk, c] = torch.matmul(pt, do).transpose(0, 1).to(q.dtype)
        del pt
        dp = torch.matmul(do, vs.transpose(1, 2).contiguous()).view(nc * G, nq, nk)
        ds = p * (dp - (p * dp).sum(2, keepdim=True))
        del dp, p
        dq[rq, hs] = (torch.matmul(ds.view(nc, G * nq, nk), ks) * scale).view(nc * G, nq, -1).transpose(0, 1).to(q.dtype)
        dst = ds.view(nc, G * nq, nk).transpose(1, 2).contiguous()
        dk[rk, c] = (torch.matmul(dst, qs) * scale).transpose(0, 1).to(q.dtype)
        del dst
        # the sums along the diagonals (seen with rows one place longer than they are, each row begins one place further back) and
        # then over the distances of every bucket
        width = nk + nq
        flat = torch.nn.functional.pad(ds, (0, nq - 1)).view(nc * G, -1)
        diag = torch.nn.functional.pad(flat, (0, nq)).view(nc * G, nq, width).sum(1)
        m = torch.arange(width, device=DEV)
        dist = torch.where(m < nk, m, m - width) - (nk - nq)
        db = (cuts[:, None] <= dist).sum(0)
        for b in range(bias.shape[0]):
            dbias[b, hs] += (diag * (db == b)).sum(1)
        del flat, ds
    return out if kind == "attend" else (out, dq, dk, dv, dbias)


def _plain_clip(state):
    total = sum((g.float() * g.float()).sum() for g in state["grads"])
    norm = torch.sqrt(total)
    coef = (state["max_norm"] / (norm + 1e-6)).clamp_max(1.0)
    coef = torch.where(torch.isfinite(norm), coef, torch.ones_like(coef))
    for g, out in zip(state["grads"], state["outs"]):
        out.copy_(g.float() * coef)
    return [norm, *state["flats"]]


def work(case):
    if case["kind"] == "clip":
        sizes = _sizes(case)
        n = sum(x for x, _ in sizes)
        return dict(bytes=2 * sum(x * (2 if t == "bf16" else 4) for x, t in sizes) + 4, flops=3 * n)
    nq, nk = _lengths(case)
    pairs = 0
    for a, b in zip(nq, nk):
        # causal: query i sees b - a + i + 1 of the keys, none if that is negative
        pairs += sum(max(0, b - a + i + 1) for i in range(a)) if case["causal"] else a * b
    H, K, D = case["heads"], case["kv_heads"], case["dim"]
    rows = 2 * D * (H * sum(nq) + K * sum(nk))           # bytes of q and k, in 16 bits
    table = 4 * H * case["buckets"]
    if case["kind"] == "attend":
        return dict(bytes=2 * rows + table, flops=4 * D * H * pairs)
    return dict(bytes=4 * rows + 2 * table, flops=14 * D * H * pairs)


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "clip":
        norm = math.sqrt(sum(float(torch.dot(g.double(), g.double())) for g in state["grads"]))
        coef = min(1.0, state["max_norm"] / (norm + 1e-6))
        flats = []
        for d in sorted({g.dtype for g in state["grads"]}, key=str):
            pieces = [g.double() * coef for g in state["grads"] if g.dtype == d]
            flats.append(torch.cat([torch.nn.functional.pad(x, (0, -len(x) % 16)) for x in pieces]))
        return [torch.tensor(norm, dtype=torch.float64, device=DEV), *flats]
    if work(case)["flops"] > 4e12:
        return None
    H, K, D = case["heads"], case["kv_heads"], case["dim"]
    G = H // K
    train = case["kind"] == "train"
    out = torch.zeros(state["q"].shape, dtype=torch.float64, device=DEV)
    grads = [torch.zeros(state[n].shape, dtype=torch.float64, device=DEV) for n in ("q", "k", "v")] if train else []
    dbias = torch.zeros(state["bias"].shape, dtype=torch.float64, device=DEV)
    edges = torch.tensor(state["cuts"], device=DEV)
    for s, (nq, nk) in enumerate(zip(state["nq"], state["nk"])):
        q0, k0 = state["q_ptr"][s], state["k_ptr"][s]
        place = torch.arange(nq, device=DEV) + (nk - nq)
        gap = torch.arange(nk, device=DEV) - place[:, None]
        bucket = torch.bucketize(gap, edges, right=True)             # how many cuts are at most the distance
        seen = gap <= 0 if case["causal"] else torch.ones_like(gap, dtype=torch.bool)
        some = seen.any(1, keepdim=True)
        for h in range(H):
            leaf = [state["q"][q0:q0 + nq, h].double(), state["k"][k0:k0 + nk, h // G].double(), state["v"][k0:k0 + nk, h // G].double()]
            leaf = [x.requires_grad_(train) for x in leaf]
            add = state["bias"][:, h].double()[bucket].requires_grad_(train)
            logit = torch.where(seen, leaf[0] @ leaf[1].T * state["scale"] + add, -math.inf)
            prob = torch.where(some, torch.softmax(torch.where(some, logit, 0.0), dim=1), 0.0)
            o = prob @ leaf[2]
            out[q0:q0 + nq, h] = o.detach()
            if train:
                d = torch.autograd.grad(o, [*leaf, add], state["dout"][q0:q0 + nq, h].double())
                grads[0][q0:q0 + nq, h] += d[0]
                grads[1][k0:k0 + nk, h // G] += d[1]
                grads[2][k0:k0 + nk, h // G] += d[2]
                dbias[:, h] += torch.stack([(d[3] * (bucket == b)).sum() for b in range(case["buckets"])])
    return (out, *grads, dbias) if train else out
