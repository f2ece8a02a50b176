"""The paged cache's calls written plainly in 64 bits, one sequence and head after the other, and how far a correct
kernel may be from them.

Bounds.  fp32 arithmetic has steps of 2^-23, so a rounding is off by at most u = 2^-24 of its result.
  logit      x = scale <q, k>: d products and sums, the factor, its place in an exponent and the exponential itself (4 roundings):
             |dx| <= dlt = scale (d + 4) u <|q|, |k|> + 4 u |x| + 4 u, maximum over what the row sees
  o          sum_j p_j v_j / sum_j p_j: each p_j off by a factor e^dlt above and below, sums of n terms by n u:
             A (2 dlt + 2 (n + 8) u), A = sum_j p_j |v_j|; bf16: each p_j also rounded (2^-8 A) and the result (2^-8 |o|)
  lse        dlt + (n + 8) u + 2 u |lse|
  weights    sum_t p_tj (dlt_t + 4 u |lse_t|) + (R + 8) u (w_j + sum_t p_tj), R rows
"""
import math

import torch

U = 2.0 ** -24


class Cache:
    """Pages, table and lengths on the CPU; kv-head h of sequence b by slots."""

    def __init__(self, k, v, table, lens, weights=None, pos=None, seen=None):
        self.k, self.v, self.table, self.lens = k, v, table, lens
        self.weights, self.pos, self.seen = weights, pos, seen
        self.page = k.shape[2]

    def where(self, b, n):
        at = torch.arange(n)
        return self.table[b].long()[at // self.page], at % self.page


def rows_of(row_start, b):
    return int(row_start[b]), int(row_start[b + 1] - row_start[b])


def _logits(c, q, row_start, b, h, g, scale, causal):
    """x, visible [g, m, n] and dlt [g, m] of a kv-head's rows."""
    n, d = int(c.lens[b]), q.shape[-1]
    r0, m = rows_of(row_start, b)
    page, off = c.where(b, n)
    K = c.k[page, h, off].double()
    Q = q[r0:r0 + m, h * g:(h + 1) * g].double().transpose(0, 1)
    x = Q @ K.t() * scale
    t = torch.arange(m)[:, None]
    vis = (torch.arange(n)[None] <= n - m + t) if causal else torch.ones((m, n), dtype=torch.bool)
    vis = vis.expand(g, m, n)
    dlt = scale * (d + 4) * U * (Q.abs() @ K.abs().t()) + 4 * U * x.abs() + 4 * U
    dlt = torch.where(vis, dlt, torch.zeros(())).amax(-1) if n else torch.zeros((g, m))
    return x.masked_fill(~vis, -math.inf), dlt.double()


def attend(c, q, row_start, h_kv, causal=True, scale=None):
    """o, lse and their bounds, NaN for rows of no sequence."""
    rows, h_q, d = q.shape
    g, scale = h_q // h_kv, scale or 1.0 / math.sqrt(d)
    o = torch.full((rows, h_q, d), math.nan, dtype=torch.float64)
    lse = torch.full((rows, h_q), math.nan, dtype=torch.float64)
    o_tol, lse_tol = torch.zeros_like(o), torch.zeros_like(lse)
    half = 2.0 ** -8 if q.dtype == torch.bfloat16 else 0.0
    for b in range(len(c.lens)):
        n = int(c.lens[b])
        r0, m = rows_of(row_start, b)
        if m == 0:
            continue
        page, off = c.where(b, n)
        for h in range(h_kv):
            x, dlt = _logits(c, q, row_start, b, h, g, scale, causal)
            V = c.v[page, h, off].double()
            l = torch.logsumexp(x, -1) if n else torch.full((g, m), -math.inf, dtype=torch.float64)
            p = torch.where(torch.isinf(l)[..., None], torch.zeros(()).double(), torch.exp(x - l[..., None]))
            y, A = p @ V, p @ V.abs()
            s = (slice(r0, r0 + m), slice(h * g, (h + 1) * g))
            o[s], lse[s] = y.transpose(0, 1), l.t()
            o_tol[s] = (A * (2 * dlt + 2 * (n + 8) * U + half)[..., None] + (half + U) * y.abs()).transpose(0, 1)
            lse_tol[s] = (dlt + (n + 8) * U + 2 * U * torch.where(torch.isinf(l), torch.zeros(()).double(), l).abs()).t()
    return o, lse, o_tol, lse_tol


def weigh(c, q, row_start, lse, h_kv, causal=True, scale=None, last=0):
    """The weights after the call and their bounds."""
    d, g = q.shape[-1], q.shape[1] // h_kv
    scale = scale or 1.0 / math.sqrt(d)
    w = c.weights.double().clone()
    tol = torch.zeros_like(w)
    for b in range(len(c.lens)):
        n = int(c.lens[b])
        r0, m = rows_of(row_start, b)
        if m == 0 or n == 0:
            continue
        page, off = c.where(b, n)
        for h in range(h_kv):
            x, dlt = _logits(c, q, row_start, b, h, g, scale, causal)
            l = lse[r0:r0 + m, h * g:(h + 1) * g].double().t()
            p = torch.where(torch.isneginf(x), torch.zeros(()).double(), torch.exp(x - l[..., None]))
            if last:
                p[:, :max(m - last, 0)] = 0
            l = torch.where(torch.isfinite(l), l, torch.zeros(()).double())
            add = p.sum((0, 1))
            w[page, h, off] += add
            tol[page, h, off] = (p * (dlt + 4 * U * l.abs())[..., None]).sum((0, 1)) + (g * m + 8) * U * (w[page, h, off] + add)
    return w, tol


def append(c, k_new, v_new, row_start):
    for b in range(len(c.lens)):
        n = int(c.lens[b])
        r0, m = rows_of(row_start, b)
        for t in range(m):
            slot = n - m + t
            if slot < 0:
                continue
            page, off = int(c.table[b, slot // c.page]), slot % c.page
            if not 0 <= page < c.k.shape[0]:
                continue
            c.k[page, :, off], c.v[page, :, off] = k_new[r0 + t], v_new[r0 + t]
            if c.weights is not None:
                c.weights[page, :, off] = 0
            if c.pos is not None:
                c.pos[page, :, off] = slot if c.seen is None else int(c.seen[b]) - m + t


def evict(c, budget, sinks=0, recent=0):
    """In place; returns src."""
    h_kv = c.k.shape[1]
    src = torch.full((len(c.lens), h_kv, budget), -1, dtype=torch.int32)
    for b in range(len(c.lens)):
        n = int(c.lens[b])
        left = min(n, budget)
        src[b, :, :left] = torch.arange(left, dtype=torch.int32)
        if n <= budget:
            continue
        page, off = c.where(b, n)
        for h in range(h_kv):
            w, pos = c.weights[page, h, off].tolist(), c.pos[page, h, off].tolist()
            safe = [p < sinks or p >= int(c.seen[b]) - recent for p in pos]
            order = sorted(range(n), key=lambda i: (not safe[i], math.inf if math.isnan(w[i]) and not safe[i] else -w[i] if not safe[i] else 0.0,
                                                    1 if math.isnan(w[i]) and not safe[i] else 0, i))
            kept = set(order[:budget])
            holes = [i for i in range(budget) if i not in kept]
            movers = [i for i in range(budget, n) if i in kept]
            for to, frm in zip(holes, movers):
                src[b, h, to] = frm
                for x in (c.k, c.v, c.weights, c.pos):
                    x[page[to], h, off[to]] = x[page[frm], h, off[frm]]
        c.lens[b] = budget
    return src
