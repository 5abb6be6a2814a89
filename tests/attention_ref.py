"""Attention over ragged rows in 64 bits on the CPU, and how far the library's results may be from it.

The bounds follow from what the library says it rounds (u, half a unit in the last place, is 2^-8 for bfloat16 and 2^-11 for float16; all
else is held in 32 bits):

  scores        32-bit sums of head_dim exact products and a product with the scale: |err S| <= eS, a few 2^-24 of scale * sum |q k| + |S|;
                a row's statistic is then off by sum_j P eS, a probability by the factor of both, and by 2^-19 for the exponential
                and the 32-bit sum of the row
  out           each probability rounded once: u sum_j P |v|, the result once: u |out|
  delta         for dq of out before its last rounding (or nearly: the difference is rounded, u^2 |out|): sum_d |dout| times that error of out;
                for dk and the bias the sum of P dP in 32 bits
  dS            P (err dP + err delta) in 32 bits, rounded once for the products with q and k: u |dS|
"""
import math

import torch

U = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16)} | {torch.float64: 0.0}
TINY = {torch.bfloat16: 1e-37, torch.float16: 2.0 ** -24, torch.float64: 0.0}     # below the smallest normal number rounding is absolute


class Reference:
    """One call's results and bounds, from the formulas."""

    def __init__(self, q, k, v, spans, causal, scale, bias=None, cuts=None, dout=None):
        """spans: (first query row, queries, first key row, keys) of every sequence.  Tensors on the CPU."""
        dt = q.dtype
        u, tiny = U[dt], TINY[dt]
        H, K, D = q.shape[1], k.shape[1], q.shape[2]
        G = H // K
        f = torch.float64
        q, k, v = q.to(f), k.to(f), v.to(f)
        self.out, self.out_tol = torch.zeros_like(q), torch.zeros_like(q)
        self.lse = torch.full((H, q.shape[0]), -math.inf, dtype=f)
        self.lse_tol = torch.zeros_like(self.lse)
        self.covered_q = torch.zeros(q.shape[0], dtype=torch.bool)
        self.covered_k = torch.zeros(k.shape[0], dtype=torch.bool)
        if dout is not None:
            g = dout.to(f)
            self.dq, self.dk, self.dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
            self.dq_tol, self.dk_tol, self.dv_tol = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
            if bias is not None:
                self.dbias = torch.zeros(bias.shape, dtype=f)
                self.dbias_tol = torch.zeros(bias.shape, dtype=f)
        edges = None if cuts is None else torch.tensor(list(cuts), dtype=torch.int64)
        for q0, nq, k0, nk in spans:
            self.covered_q[q0:q0 + nq] = True
            self.covered_k[k0:k0 + nk] = True
            if nq == 0:
                continue
            t = torch.arange(nk)[None, :] - (torch.arange(nq)[:, None] + (nk - nq))
            seen = t <= 0 if causal else torch.ones_like(t, dtype=torch.bool)
            b = None if edges is None else torch.bucketize(t, edges, right=True)
            for h in range(H):
                c = h // G
                qs, ks, vs = q[q0:q0 + nq, h], k[k0:k0 + nk, c], v[k0:k0 + nk, c]
                s = qs @ ks.T * scale
                es = (abs(scale) * (qs.abs() @ ks.abs().T) * (D + 8) * 2.0 ** -24 + s.abs() * 2.0 ** -22) + 2.0 ** -22
                if bias is not None:
                    add = bias[:, h].to(f)[b]
                    s = s + add
                    es = es + add.abs() * 2.0 ** -22
                keep = seen & (s > -math.inf)                  # a bias of -inf shuts its bucket out
                s, es = s.masked_fill(~keep, -math.inf), es.masked_fill(~keep, 0.0)
                some = keep.any(1)
                lse = torch.logsumexp(s, 1) if nk else torch.full((nq,), -math.inf, dtype=f)
                p = torch.where(keep, torch.exp(s - torch.where(some, lse, 0.0)[:, None]), 0.0)
                elog = (p * es).sum(1, keepdim=True)           # of the row's statistic, to first order
                ep = p * (1.1 * (es + elog) + 2.0 ** -19)      # of a probability
                self.lse[h, q0:q0 + nq] = torch.where(some, lse, -math.inf)
                self.lse_tol[h, q0:q0 + nq] = 1.1 * elog[:, 0] + 2.0 ** -19 * (1 + torch.where(some, lse.abs(), 0.0))
                o = p @ vs
                spread = p @ vs.abs()
                self.out[q0:q0 + nq, h] = o
                self.out_tol[q0:q0 + nq, h] = u * (1.01 * spread + 1.01 * o.abs()) + ep @ vs.abs() + tiny * (1 + spread)
                if dout is None:
                    continue
                gs = g[q0:q0 + nq, h]
                dp = gs @ vs.T
                delta = (p * dp).sum(1, keepdim=True)
                ds = p * (dp - delta)
                edp = (gs.abs() @ vs.abs().T) * (D + 2) * 2.0 ** -24
                acc = 2.0 ** -24 * (max(nq, nk) + 8)           # 32-bit sums over the rows
                e_out = self.out_tol[q0:q0 + nq, h] - u * o.abs() + u * u * o.abs()
                edelta_q = (gs.abs() * (e_out + o.abs() * (D + 2) * 2.0 ** -24)).sum(1, keepdim=True)
                # the row sum of P (dP - delta'), added to delta': sum P dP, and (1 - sum P) delta' on top
                edelta = (p * edp + ep * (dp.abs() + 2 * delta.abs()) + acc * (p * (dp.abs() + delta.abs()))).sum(1, keepdim=True) + acc * delta.abs()

                def of_ds(ed):
                    return p * (edp + ed) + ep * (dp.abs() + delta.abs() + ed) + 2.0 ** -23 * ds.abs()

                eds, eds_q = of_ds(edelta), of_ds(edelta_q)
                rds, rds_q = (e + 1.01 * u * (ds.abs() + e) + tiny for e in (eds, eds_q))
                rp = ep + 1.01 * u * p + tiny
                self.dq[q0:q0 + nq, h] = ds @ ks * scale
                self.dq_tol[q0:q0 + nq, h] = abs(scale) * ((rds_q + acc * ds.abs()) @ ks.abs())
                self.dk[k0:k0 + nk, c] += ds.T @ qs * scale
                self.dk_tol[k0:k0 + nk, c] += abs(scale) * ((rds + acc * G * ds.abs()).T @ qs.abs())
                self.dv[k0:k0 + nk, c] += p.T @ gs
                self.dv_tol[k0:k0 + nk, c] += (rp + acc * G * p).T @ gs.abs()
                if bias is not None:
                    self.dbias[:, h].index_add_(0, b.flatten(), ds.flatten())
                    self.dbias_tol[:, h].index_add_(0, b.flatten(), (eds + acc * 4 * ds.abs()).flatten())
        if dout is not None:
            for x in (("dq", "dk", "dv")):
                val, tol = getattr(self, x), getattr(self, x + "_tol")
                tol += 1.01 * u * val.abs() + tiny
            if bias is not None:
                self.dbias_tol += 2.0 ** -20 * self.dbias.abs() + 1e-30


def rows_of(counts):
    ptr = [0]
    for c in counts:
        ptr.append(ptr[-1] + c)
    return ptr


def close(got, want, tol, what):
    got = got.detach().cpu().double()
    bad = ~((got - want).abs() <= tol) & ~(got == want)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {((got - want).abs() / tol.clamp_min(1e-300))[bad].max():.3g} "
                           f"times the bound at {bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]}")
