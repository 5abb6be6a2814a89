"""Plain 64-bit forms of the operators around a tower (on the CPU), and bounds of what 32-bit arithmetic may be off by."""
import math

import torch

U = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
U32 = 2.0 ** -24
# what the matrix units' host, the vector unit's sine and cosine of a fraction of a revolution, may be off by
TURN = 2.0 ** -18


def lookup(table, ids, scale):
    rows = table.shape[0]
    out = torch.zeros(*ids.shape, table.shape[1], dtype=torch.float64)
    for at in torch.cartesian_prod(*[torch.arange(n) for n in ids.shape]).view(-1, ids.dim()):
        v = int(ids[tuple(at)])
        if 0 <= v < rows:
            out[tuple(at)] = table[v].double() * scale
    return out


def lookup_gradient(dout, ids, rows, scale, old=None):
    """(gradient, bound of its error before the last rounding)."""
    flat, d = ids.flatten().long(), dout.reshape(ids.numel(), -1).double()
    inside = (flat >= 0) & (flat < rows)
    total = torch.zeros(rows, d.shape[1], dtype=torch.float64)
    size, count = torch.zeros_like(total), torch.zeros(rows, 1, dtype=torch.float64)
    total.index_add_(0, flat[inside], d[inside])
    size.index_add_(0, flat[inside], d[inside].abs())
    count.index_add_(0, flat[inside], torch.ones(int(inside.sum()), 1, dtype=torch.float64))
    got = total * scale
    bound = abs(scale) * (count + 1) * U32 * size          # any order of n terms: n - 1 roundings of partial sums; the product
    if old is not None:
        got = torch.where(count > 0, got + old.double(), old.double())
        bound = bound + U32 * got.abs()
    return got, bound


def places(rows, q_ptr=None, k_ptr=None, k_len=None, n_seq=1, store_rows=None):
    """For every row (sequence's rows or not, place, row of the store or -1), by going through the sequences."""
    there, place, to = [False] * rows, [0] * rows, [-1] * rows
    if q_ptr is None:
        q_ptr = [s * (rows // n_seq) for s in range(n_seq + 1)]
    for s in range(len(q_ptr) - 1):
        q0, q1 = q_ptr[s], q_ptr[s + 1]
        nq = q1 - q0
        slot, room = 0, nq
        if k_ptr is not None or k_len is not None:
            if k_ptr is not None:
                slot, room = k_ptr[s], k_ptr[s + 1] - k_ptr[s]
            elif store_rows is not None:
                room = store_rows // (len(q_ptr) - 1)
                slot = s * room
            else:
                room = 1 << 30
            if k_len is not None:
                room = min(room, k_len[s])
        for i in range(nq):
            there[q0 + i] = True
            place[q0 + i] = i + room - nq
            if 0 <= place[q0 + i] < room:
                to[q0 + i] = slot + place[q0 + i]
    return torch.tensor(there), torch.tensor(place, dtype=torch.int64), torch.tensor(to, dtype=torch.int64)


def _turn(y, position, turns, halves, sign=1.0):
    """y [rows][heads][dim], and the length of each element's pair."""
    r = 2 * len(turns)
    y, size = y.clone(), y.abs()
    whole = position.double()[:, None, None] * turns
    angle = sign * (whole - whole.round()) * 2 * math.pi
    at = torch.arange(r)
    a, b = (at[:r // 2], at[r // 2:]) if halves else (at[0::2], at[1::2])
    x, z = y[..., a], y[..., b]
    y[..., a], y[..., b] = x * angle.cos() - z * angle.sin(), z * angle.cos() + x * angle.sin()
    size[..., a] = size[..., b] = torch.hypot(x, z)
    return y, size


def rotate(x, weight, turns, position, there, eps, halves):
    """(result, bound of its error before the last rounding)."""
    d = x.shape[-1]
    x = torch.where(there[:, None, None], x.double(), 0.0)
    s = torch.where(there[:, None, None], 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps), 0.0)
    y, size = _turn(x * s * weight.double(), position, turns, halves)
    # a sum of d squares, its root and quotient, two products, and two with the sine and cosine
    return y, size * ((d / 2 + 16) * U32 + TURN)


def rotate_gradient(dout, x, weight, turns, position, there, eps, halves):
    """(dx, its bound before the last rounding, dweight, its bound)."""
    d = x.shape[-1]
    x, g = (torch.where(there[:, None, None], t.double(), 0.0) for t in (x, dout))
    w = weight.double()
    s = torch.where(there[:, None, None], 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps), 0.0)
    g, size = _turn(g, position, turns, halves, -1.0)
    u = g * w
    dx = s * (u - x * s * s * (x * u).mean(-1, keepdim=True))
    each = (2 * d + 32) * U32 + TURN
    bound = each * s * (size * w.abs() + x.abs() * s * s * (x.abs() * size * w.abs()).mean(-1, keepdim=True))
    n = x.shape[0] * x.shape[1]
    return dx, bound, (g * x * s).sum((0, 1)), ((n * U32 + each) * size * x.abs() * s).sum((0, 1))


def newton_schulz(g, steps, coefficients):
    """(result, a bound of its error in the Frobenius norm before the last rounding).

    Every step leaves an error of a few 2^-22 of its X (operands of 22 bits, three products, sums in 32 bits of which the roundings add up like their
    root), and the steps behind it take that on: a function of the singular values takes an error on by at most its largest difference quotient
    between any two of them, or between one and another's negative."""
    a, b, c = coefficients
    x = g.double()
    norm = torch.linalg.vector_norm(x)
    if float(norm) == 0.0:
        return x, 0.0
    x = x / norm
    u, s, vt = torch.linalg.svd(x, full_matrices=False)
    values = [s]
    for _ in range(steps):
        t = values[-1]
        values.append(t * (a + b * t ** 2 + c * t ** 4))
    bound = 0.0
    per_step = (8 + math.sqrt(max(g.shape))) * 2.0 ** -22 * (abs(a) + abs(b) + abs(c))
    for k in range(steps + 1):
        f, t = values[-1], values[k]
        if k == steps:
            worst = 1.0
        else:
            slope = torch.ones_like(t)
            for y in values[k:-1]:
                slope = slope * (a + 3 * b * y ** 2 + 5 * c * y ** 4)
            dt, df = t[:, None] - t, f[:, None] - f
            apart = dt.abs() > 1e-6
            worst = max(float(slope.abs().max()), float(torch.where(apart, df / torch.where(apart, dt, 1.0), 0.0).abs().max()),
                        float(((f[:, None] + f) / (t[:, None] + t).clamp_min(1e-12)).abs().max()))
            if min(g.shape) < max(g.shape):
                worst = max(worst, float((f / t.clamp_min(1e-12)).abs().max()))
        bound += worst * per_step * float(torch.linalg.vector_norm(t))
    return u @ torch.diag(values[-1]) @ vt, bound
