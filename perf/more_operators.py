"""The operators around an attention tower over histories of events, as workloads.

What a tower needs besides its attention and the clipping of its gradients.  The operators:

  embed        the events' rows of an embedding table, times a factor; ids outside the table give zeros
  embed_train  the same and the table's gradient: the sum of the gradients of all places that hold a row's id
  heads        norms of the queries and keys of every head, and their rotation by position: scoring, with the keys (and the values)
               written into the store that attention reads, or packed as they came
  heads_train  the same packed, and its backward pass: gradients of q, k and of the norms' weights
  ortho        updates of weight matrices, orthogonalised by Newton-Schulz products

A case is a dict of plain values.  For embed and embed_train: places ids over a table of rows x width, ids as frequent as 1 / (rank + 1)
** skew, a share `pad` of them outside the table; table, out and grad are types.  For heads and heads_train: seqs histories, whose
numbers of new rows lie in q_lo..q_hi, behind past_lo..past_hi stored ones (scoring with `store`); heads, kv_heads, dim, and `turned` of
the dim elements rotated, as neighbouring pairs or as halves; `far`: explicit positions up to it, 0: places in the history.  For
ortho: a list of shapes, each with how often it comes, as text "m x n * count, ...".
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6
STEPS, COEFFICIENTS = 5, (3.4445, -4.7750, 2.0315)


def _embed(name, kind, places, rows, width, table="f32", out="bf16", grad="f32", skew=1.0, pad=0.0, wide=True):
    return dict(name=name, kind=kind, places=places, rows=rows, width=width, table=table, out=out, grad=grad, skew=skew, pad=pad, wide=wide)


def _heads(name, kind, seqs, q_lo, q_hi, heads, kv_heads, dim, turned, dtype="bf16", halves=True, store=False, past_lo=0, past_hi=0, far=0,
           lengths=0):
    return dict(name=name, kind=kind, seqs=seqs, q_lo=q_lo, q_hi=q_hi, heads=heads, kv_heads=kv_heads, dim=dim, turned=turned, dtype=dtype,
                halves=halves, store=store, past_lo=past_lo, past_hi=past_hi, far=far, lengths=lengths)


def _ortho(name, shapes, dtype):
    return dict(name=name, kind="ortho", shapes=shapes, dtype=dtype)


def listed():
    return [
        # the smallest call: one new event for each of 48 rows
        _embed("embed_new_events", "embed", 48, 5_000, 512, table="bf16"),
        # a batch of long histories over a large vocabulary of events, some places padded; the table in 32 bits
        _embed("embed_long", "embed", 65_536, 120_000, 2_048, pad=0.05),
        # a training step of a small tower: some 2000 events of 40 kinds
        _embed("embed_train_small", "embed_train", 1_999, 40, 64, out="f32", skew=0.5),
        # one of the example's size: 900,000 events of 12 kinds
        _embed("embed_train_kinds", "embed_train", 900_000, 12, 64, skew=0.3),
        # a large one: very unequal frequencies, most rows of the table untouched, ids in 32 bits
        _embed("embed_train_large", "embed_train", 32_768, 120_000, 2_048, table="bf16", skew=1.1, pad=0.02, wide=False),
        # new events, one a row, appended to the store
        _heads("heads_new_event", "heads", 48, 1, 1, 8, 2, 64, 64, store=True, past_lo=30, past_hi=500),
        # whole histories into the store
        _heads("heads_histories", "heads", 24, 100, 1_500, 16, 8, 128, 128, store=True),
        # a head size that is no power of two, turned in part, as pairs, at explicit far positions
        _heads("heads_train_odd", "heads_train", 5, 301, 777, 6, 2, 80, 32, dtype="f16", halves=False, far=1_000_000),
        # the largest training batch
        _heads("heads_train_long", "heads_train", 8, 3_500, 4_096, 32, 8, 128, 128),
        # the matrices of a small tower
        _ortho("ortho_tower", "64 x 256 * 1, 128 x 64 * 2, 40 x 64 * 1", "f32"),
        # of an ordinary model: some layers' projections, odd sizes among them, all in one call
        _ortho("ortho_model", "512 x 1536 * 6, 512 x 512 * 6, 512 x 2048 * 6, 2048 x 512 * 6, 777 x 1001 * 2", "bf16"),
        # of a large one
        _ortho("ortho_large", "4096 x 4096 * 1, 1024 x 4096 * 2, 4096 x 8192 * 1", "f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "embed_train", "embed_train", "heads", "heads", "heads_train", "heads_train", "ortho", "ortho"])
    if kind.startswith("embed"):
        width = _log_int(rng, 4, 2_048)
        if rng.random() < 0.7:
            width = max(8, width // 8 * 8)
        places = _log_int(rng, 1, min(900_000, 32_768 * 2_048 // width))
        rows = _log_int(rng, 2, min(120_000, 120_000 * 2_048 // width))
        return _embed("", kind, places, rows, width, rng.choice(["f32", "bf16", "f16"]), rng.choice(["f32", "bf16", "bf16", "f16"]),
                      rng.choice(["f32", "f32", "bf16"]), rng.choice([0.0, 0.5, 1.0, 1.3]), rng.choice([0.0, 0.0, 0.1]), rng.random() < 0.5)
    if kind.startswith("heads"):
        kv_heads = rng.choice([1, 2, 4, 5, 8])
        heads = kv_heads * rng.choice([1, 1, 2, 4])
        dim = rng.choice([8, 16, 32, 40, 64, 64, 80, 96, 128, 128])
        turned = dim if rng.random() < 0.6 else rng.randrange(8, dim + 1, 8)
        dtype = rng.choice(["bf16", "bf16", "f16"])
        store = kind == "heads" and rng.random() < 0.7
        q_hi = 1 if store and rng.random() < 0.3 else _log_int(rng, 2, 3_000)
        seqs = max(1, min(64, _log_int(rng, 1, 64), 24_000 // q_hi))
        past = _log_int(rng, 1, 1_000) if store else 0
        far = 0 if store or rng.random() < 0.6 else _log_int(rng, 100, 1_000_000)
        return _heads("", kind, seqs, max(1, q_hi // 5), q_hi, heads, kv_heads, dim, turned, dtype, rng.random() < 0.6, store, past // 3, past, far,
                      rng.randrange(1 << 20))
    shapes, left = [], 4.0e11
    for _ in range(rng.randint(1, 5)):
        m, n = _log_int(rng, 8, 2_500), _log_int(rng, 8, 2_500)
        count = rng.randint(1, 6)
        cost = min(m, n) ** 2 * max(m, n) * 30.0
        if cost * count <= left:
            left -= cost * count
            shapes.append(f"{m} x {n} * {count}")
    return _ortho("", ", ".join(shapes) or "64 x 40 * 1", rng.choice(["f32", "bf16", "bf16", "f16"]))


def _lengths(case):
    """The new rows of every history, and the stored ones before them: a property of the case."""
    rng = random.Random(f"{case['lengths']} {case['seqs']} {case['q_lo']} {case['q_hi']}")
    new = [rng.randint(case["q_lo"], case["q_hi"]) for _ in range(case["seqs"])]
    return new, [rng.randint(case["past_lo"], case["past_hi"]) for _ in range(case["seqs"])]


def _shapes(case):
    out = []
    for part in case["shapes"].split(","):
        shape, count = part.split("*")
        m, n = shape.split("x")
        out += [(int(m), int(n))] * int(count)
    return out


def _rng(seed, salt):
    return torch.Generator(device=DEV).manual_seed(seed * 7919 + salt)


def _ptr(counts):
    p = [0]
    for c in counts:
        p.append(p[-1] + c)
    return p


def prepare(case, seed):
    return {"e": _prepare_embed, "h": _prepare_heads, "o": _prepare_ortho}[case["kind"][0]](case, _rng(seed, 1))


def _prepare_embed(case, r):
    places, rows, width = case["places"], case["rows"], case["width"]
    # ids by their frequency, the frequent ones anywhere in the table
    share = (torch.arange(1, rows + 1, device=DEV, dtype=torch.float64)) ** -case["skew"]
    edge = share.cumsum(0)
    rank = torch.searchsorted(edge, torch.rand(places, generator=r, device=DEV, dtype=torch.float64) * edge[-1]).clamp_max(rows - 1)
    ids = torch.randperm(rows, generator=r, device=DEV)[rank]
    ids = torch.where(torch.rand(places, generator=r, device=DEV) < case["pad"], torch.full_like(ids, -1), ids)
    state = dict(case=case, ids=ids if case["wide"] else ids.int(), scale=math.sqrt(width),
                 table=(torch.randn(rows, width, generator=r, device=DEV) * width ** -0.5).to(TYPES[case["table"]]))
    if case["kind"] == "embed_train":
        state["dout"] = (torch.randn(places, width, generator=r, device=DEV) / 64).to(TYPES[case["out"]])
    if own:
        state["ctx"] = _context()
    return state


def _prepare_heads(case, r):
    new, past = _lengths(case)
    H, K, D, dt = case["heads"], case["kv_heads"], case["dim"], TYPES[case["dtype"]]
    rows = sum(new)
    # parts of one projection's output; heads of different size, as a projection makes them
    size = torch.exp(torch.randn(H + 2 * K, 1, generator=r, device=DEV) * 0.7)
    q, k, v = (torch.randn(rows, H + 2 * K, D, generator=r, device=DEV) * size).to(dt).split([H, K, K], dim=1)
    q_ptr = torch.tensor(_ptr(new), device=DEV)
    i = torch.arange(0, case["turned"], 2, device=DEV, dtype=torch.float64) / case["turned"]
    state = dict(case=case, q=q, k=k, v=v, new=new, past=past, q_ptr=q_ptr, turns=10_000.0 ** -i / (2 * math.pi),
                 q_weight=1 + 0.2 * torch.randn(D, generator=r, device=DEV), k_weight=1 + 0.2 * torch.randn(D, generator=r, device=DEV))
    if case["far"]:
        state["positions"] = torch.randint(0, case["far"] + 1, (rows,), generator=r, device=DEV, dtype=torch.int32)
    if case["store"]:
        room = [a + b + (a + b) // 8 + 16 for a, b in zip(new, past)]
        state["k_ptr"] = torch.tensor(_ptr(room), device=DEV)
        state["k_len"] = torch.tensor([a + b for a, b in zip(new, past)], dtype=torch.int32, device=DEV)
        state["k_store"], state["v_store"] = (torch.randn(sum(room), K, D, generator=r, device=DEV).to(dt) for _ in range(2))
    if case["kind"] == "heads_train":
        state["dq_out"] = torch.randn(rows, H, D, generator=r, device=DEV).to(dt)
        state["dk_out"] = torch.randn(rows, K, D, generator=r, device=DEV).to(dt)
    if own:
        state["ctx"] = _context()
        state["args"] = dict(halves=case["halves"], eps=EPS)
        if case["far"]:
            state["args"]["positions"] = state["positions"]
        elif case["q_hi"] > 1:
            state["args"]["q_ptr"] = q_ptr
        if case["store"]:
            state["args"].update(k_ptr=state["k_ptr"], k_len=state["k_len"])
            state["store"] = dict(v=v, k_out=state["k_store"], v_out=state["v_store"])
        elif not case["far"] and case["q_hi"] == 1:
            state["args"]["q_ptr"] = q_ptr
    return state


def _prepare_ortho(case, r):
    # averaged gradients: a few strong directions, and many weak ones
    updates = []
    for m, n in _shapes(case):
        few = max(1, min(m, n) // 16)
        g = torch.randn(m, few, generator=r, device=DEV) @ torch.randn(few, n, generator=r, device=DEV)
        updates.append(((g + torch.randn(m, n, generator=r, device=DEV)) * 1e-3).to(TYPES[case["dtype"]]))
    outs = [torch.zeros_like(u) for u in updates]
    scales = [max(1.0, m / n) ** 0.5 for m, n in _shapes(case)]
    state = dict(case=case, updates=updates, outs=outs, scales=scales)
    if own:
        state["ctx"] = _context()
        state["plan"] = state["ctx"].matrix_list(updates, outs, scales=scales)
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
    kind = state["case"]["kind"]
    if own:
        return _run_own(state, kind)
    return {"e": _plain_embed, "h": _plain_heads, "o": _plain_ortho}[kind[0]](state)


def _run_own(state, kind):
    ctx, case = state["ctx"], state["case"]
    if kind == "ortho":
        ctx.orthogonalise(state["plan"], steps=STEPS, coefficients=COEFFICIENTS)
        return state["outs"]
    if kind.startswith("embed"):
        out = ctx.embedding(state["table"], state["ids"], scale=state["scale"], dtype=TYPES[case["out"]])
        if kind == "embed":
            return out
        return out, ctx.embedding_backward(state["dout"], state["ids"], case["rows"], scale=state["scale"], dtype=TYPES[case["grad"]])
    operands = state["q"], state["k"], state["q_weight"], state["k_weight"], state["turns"]
    if case["store"]:
        q_out, k_store, v_store = ctx.norm_rotate(*operands, **state["args"], **state["store"])
        return q_out, k_store, v_store
    out = ctx.norm_rotate(*operands, **state["args"])
    if kind == "heads":
        return out
    return (*out, *ctx.norm_rotate_backward(state["dq_out"], state["dk_out"], *operands, **state["args"]))


def _plain_embed(state):
    case, ids = state["case"], state["ids"].long()
    seen = (ids >= 0) & (ids < case["rows"])
    at = torch.where(seen, ids, torch.zeros_like(ids))
    out = (state["table"][at].float() * state["scale"]).masked_fill(~seen[:, None], 0.0).to(TYPES[case["out"]])
    if case["kind"] == "embed":
        return out
    long = case["places"] > 256 * case["rows"]
    if long and case["rows"] <= 64:
        total = torch.stack([torch.where((ids == v)[:, None], state["dout"], 0).sum(0, dtype=torch.float64) for v in range(case["rows"])])
    else:
        wide = torch.float64 if long else torch.float32
        total = torch.zeros(case["rows"], case["width"], dtype=wide, device=DEV)
        total.index_add_(0, at, state["dout"].to(wide).masked_fill(~seen[:, None], 0.0))
    return out, (total * state["scale"]).to(TYPES[case["grad"]])


def _places(state):
    """The position of every row, in 64 bits."""
    if "positions" in state:
        return state["positions"].long()
    new = torch.tensor(state["new"], device=DEV)
    begin = state["q_ptr"][:-1] - torch.tensor(state["past"], device=DEV)
    return torch.arange(len(state["q"]), device=DEV) - torch.repeat_interleave(begin, new)


def _pairs(x, turned, halves):
    """The two elements of every pair, and the rest."""
    if halves:
        return x[..., :turned // 2], x[..., turned // 2:turned], x[..., turned:]
    return x[..., 0:turned:2], x[..., 1:turned:2], x[..., turned:]


def _joined(a, b, rest, halves):
    return torch.cat([a, b, rest] if halves else [torch.stack([a, b], dim=-1).flatten(-2), rest], dim=-1)


def _plain_heads(state):
    case = state["case"]
    turned, halves, dt = case["turned"], case["halves"], TYPES[case["dtype"]]
    at = _places(state)
    angle = (at.double()[:, None] * state["turns"]).remainder(1.0) * (2 * math.pi)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def forward(x, w):
        x = x.float()
        s = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        a, b, rest = _pairs(x * s * w, turned, halves)
        return _joined(a * cos - b * sin, b * cos + a * sin, rest, halves).to(dt)

    def backward(d, x, w):
        x = x.float()
        s = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        a, b, rest = _pairs(d.float(), turned, halves)
        g = _joined(a * cos + b * sin, b * cos - a * sin, rest, halves)
        u = g * w
        dx = s * (u - x * (s * s * (x * u).mean(-1, keepdim=True)))
        return dx.to(dt), (g * x * s).sum((0, 1), dtype=torch.float64).float()

    q_out, k_out = forward(state["q"], state["q_weight"]), forward(state["k"], state["k_weight"])
    if case["store"]:
        row = torch.repeat_interleave(state["k_ptr"][:-1], torch.tensor(state["new"], device=DEV)) + at
        state["k_store"][row], state["v_store"][row] = k_out, state["v"]
        return q_out, state["k_store"], state["v_store"]
    if case["kind"] == "heads":
        return q_out, k_out
    dq, dqw = backward(state["dq_out"], state["q"], state["q_weight"])
    dk, dkw = backward(state["dk_out"], state["k"], state["k_weight"])
    return q_out, k_out, dq, dk, dqw, dkw


def _plain_ortho(state):
    a, b, c = COEFFICIENTS
    for g, out, scale in zip(state["updates"], state["outs"], state["scales"]):
        x = g.float()
        x = x / (x.double() * x.double()).sum().sqrt().clamp_min(1e-30).float()
        tall = x.shape[0] > x.shape[1]
        x = x.t().contiguous() if tall else x
        for _ in range(STEPS):
            gram = x @ x.t()
            x = a * x + (b * gram + c * (gram @ gram)) @ x
        out.copy_((x.t() if tall else x) * scale)
    return state["outs"]


def work(case):
    if case["kind"] == "ortho":
        elements = flops = 0
        for m, n in _shapes(case):
            p, wide = min(m, n), max(m, n)
            elements += m * n
            # a step: X X^T and its square are symmetric, half of each; B X; the last step is a step like the others
            flops += STEPS * (p * p * wide + p * p * p + 2 * p * p * wide)
        return dict(bytes=2 * elements * SIZE[case["dtype"]], flops=flops)
    if case["kind"].startswith("embed"):
        places, rows, width = case["places"], case["rows"], case["width"]
        of_id = 8 if case["wide"] else 4
        # rows that several places share are read once (as many as such draws hit on average), padded places read none
        share = torch.arange(1, rows + 1, dtype=torch.float64) ** -case["skew"]
        hit = float((-torch.expm1(-places * (1 - case["pad"]) * share / share.sum())).sum())
        moved = places * of_id + int(hit) * width * SIZE[case["table"]] + places * width * SIZE[case["out"]]
        if case["kind"] == "embed":
            return dict(bytes=moved, flops=places * width)
        return dict(bytes=moved + places * width * SIZE[case["out"]] + rows * width * SIZE[case["grad"]], flops=2 * places * width)
    rows = sum(_lengths(case)[0])
    H, K, D = case["heads"], case["kv_heads"], case["dim"]
    forward = 2 * rows * (H + K) * D * 2 + (2 * rows * K * D * 2 if case["store"] else 0)
    flops = rows * (H + K) * D * 7
    if case["kind"] == "heads":
        return dict(bytes=forward, flops=flops)
    # q and k once for both directions, then the outputs, their gradients and those of q and k
    return dict(bytes=4 * rows * (H + K) * D * 2, flops=3 * flops)


def exact(case, seed):
    state = prepare(case, seed)
    return {"e": _exact_embed, "h": _exact_heads, "o": _exact_ortho}[case["kind"][0]](case, state)


def _exact_embed(case, state):
    ids = state["ids"].long()
    rows, width = case["rows"], case["width"]
    # one row more, of zeros, for ids outside the table
    where = torch.where((ids < 0) | (ids >= rows), rows, ids)
    out = torch.cat([state["table"].double() * state["scale"], torch.zeros(1, width, dtype=torch.float64, device=DEV)])[where]
    if case["kind"] == "embed":
        return out
    # sums of stretches of the sorted places, as differences of running sums within blocks of columns
    order = torch.argsort(where, stable=True)
    edges = torch.searchsorted(where[order], torch.arange(rows + 1, device=DEV))
    grad = torch.empty(rows, width, dtype=torch.float64, device=DEV)
    for c in range(0, width, 256):
        run = torch.nn.functional.pad(state["dout"][order, c:c + 256].double().cumsum(0), (0, 0, 1, 0))
        grad[:, c:c + 256] = (run[edges[1:]] - run[edges[:-1]]) * state["scale"]
    return out, grad


def _exact_heads(case, state):
    turned = case["turned"]
    place = []
    for s, (n, before) in enumerate(zip(state["new"], state["past"])):
        place += range(before, before + n)
    place = state["positions"].double() if case["far"] else torch.tensor(place, device=DEV, dtype=torch.float64)
    whole = place[:, None] * state["turns"]
    unit = torch.polar(torch.ones_like(whole), (whole - whole.round()) * (2 * math.pi))[:, None]
    cols = torch.arange(turned, device=DEV)
    cols = cols.view(2, -1).t() if case["halves"] else cols.view(-1, 2)           # the elements of every pair

    def turn(y, by):
        z = torch.complex(y[..., cols[:, 0]], y[..., cols[:, 1]]) * by
        y = y.clone()
        y[..., cols[:, 0]], y[..., cols[:, 1]] = z.real, z.imag
        return y

    train = case["kind"] == "heads_train"
    outs, grads, weights = [], [], []
    for name in ("q", "k"):
        # in blocks of rows, so that autograd's copies stay small
        parts, of_x, of_w = [], [], torch.zeros(case["dim"], dtype=torch.float64, device=DEV)
        for r in range(0, len(place), 4096):
            x = state[name][r:r + 4096].double().requires_grad_(train)
            w = state[name + "_weight"].double().requires_grad_(train)
            with torch.set_grad_enabled(train):
                y = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["dim"] + EPS) * w
            parts.append(turn(y.detach(), unit[r:r + 4096]))
            if train:
                back = turn(state[f"d{name}_out"][r:r + 4096].double(), unit[r:r + 4096].conj())
                dx, dw = torch.autograd.grad(y, (x, w), back)
                of_x.append(dx)
                of_w += dw
        outs.append(torch.cat(parts))
        if train:
            grads.append(torch.cat(of_x))
            weights.append(of_w)
    if case["store"]:
        k_store, v_store = state["k_store"].double(), state["v_store"].double()
        r = 0
        for s, (n, before) in enumerate(zip(state["new"], state["past"])):
            first = int(state["k_ptr"][s]) + before
            k_store[first:first + n], v_store[first:first + n] = outs[1][r:r + n], state["v"][r:r + n].double()
            r += n
        return outs[0], k_store, v_store
    return (*outs, *grads, *weights)


def _exact_ortho(case, state):
    a, b, c = COEFFICIENTS
    result = []
    for g, scale in zip(state["updates"], state["scales"]):
        x = g.double()
        x = x / torch.linalg.vector_norm(x)
        tall = x.shape[0] > x.shape[1]
        gram = x.t() @ x if tall else x @ x.t()
        # every step multiplies by a polynomial of one symmetric matrix, which all of them commute with
        eye = torch.eye(len(gram), dtype=torch.float64, device=DEV)
        total = eye
        for _ in range(STEPS):
            factor = a * eye + b * gram + c * (gram @ gram)
            total = factor @ total
            gram = factor @ gram @ factor
        result.append((x @ total if tall else total @ x) * scale)
    return result
