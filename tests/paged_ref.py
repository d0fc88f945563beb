"""Plain 64-bit forms of the paged key/value cache operations (CPU, one sequence and head at a time), with elementwise error
bounds counted in roundings of half a step."""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # half a step relative to the value


def make_cache(g, dtype, kv, dh, page, lens, slack_pages=2, fill=float("nan")):
    """Pages in random order; slots behind a sequence's tokens hold `fill`.  Returns k, v, table (max_pages leaves one spare)."""
    mp = max(1, (max(lens) + page - 1) // page) + 1
    need = sum((n + page - 1) // page for n in lens) + slack_pages
    k = torch.full((need, kv, page, dh), fill, dtype=torch.float32)
    v = torch.full((need, kv, page, dh), fill, dtype=torch.float32)
    order = torch.randperm(need, generator=g)
    table = torch.full((len(lens), mp), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(lens):
        for c in range((n + page - 1) // page):
            p = int(order[at]); at += 1
            table[b, c] = p
            m = min(page, n - c * page)
            k[p, :, :m] = torch.randn((kv, m, dh), generator=g)
            v[p, :, :m] = torch.randn((kv, m, dh), generator=g)
    return k.to(dtype), v.to(dtype), table


def tokens(pages, table, b, n):
    """[kv, n, dh] of the first n slots of sequence b, in 64 bits."""
    page = pages.shape[2]
    ids = table[b, :(n + page - 1) // page].long()
    x = pages[ids].double()                                    # [c, kv, page, dh]
    return x.permute(1, 0, 2, 3).reshape(pages.shape[1], -1, pages.shape[3])[:, :n]


def attention(q, k, v, table, lens, starts, pos=None, scale=None, softcap=0.0, window=0, slopes=None, cap_rel=None):
    """(out, bound of out, weights per sequence, bound of the weights) in 64 bits.  cap_rel: a bound of the capping's error relative
    to the capped score, where it is not one relative to the cap."""
    H, dh = q.shape[1], q.shape[2]
    kv = k.shape[1]
    G = H // kv
    scale = dh ** -0.5 if scale is None else scale
    u = U[q.dtype]
    f = 2.0 ** -24
    out = torch.zeros(q.shape, dtype=torch.float64)
    tol = torch.zeros(q.shape, dtype=torch.float64)
    ws, wt = [], []
    for b, n in enumerate(lens):
        lo, hi = starts[b], starts[b + 1]
        nq = hi - lo
        w = torch.zeros(n, dtype=torch.float64)
        wtol = torch.zeros(n, dtype=torch.float64)
        if nq and n:
            kk, vv = tokens(k, table, b, n), tokens(v, table, b, n)
            slot = torch.arange(n - nq, n)
            p_ = (pos[b, :n] if pos is not None else torch.arange(n)).double()
            tpos = torch.where(slot >= 0, p_[slot.clamp(min=0)], slot.double())
            away = tpos[:, None] - p_[None, :]
            seen = torch.arange(n)[None, :] <= slot[:, None]
            if window:
                seen = seen & (away < window)
            for h in range(H):
                qh = q[lo:hi, h].double()
                x = qh @ kk[h // G].t() * scale
                mag = qh.abs() @ kk[h // G].abs().t() * scale       # what the roundings of the product scale with
                dx = (dh + 8) * f * mag
                if softcap:
                    x = softcap * torch.tanh(x / softcap)
                    # one exponential, one quotient, values up to 2 * softcap
                    dx = dx + (softcap * 2.0 ** -21 if cap_rel is None else cap_rel * x.abs())
                if slopes is not None:
                    bias = slopes[h].double() * away
                    x = x - bias
                    dx = dx + 4 * f * bias.abs()
                x = x.masked_fill(~seen, -math.inf)
                top = x.amax(1, keepdim=True)
                e = torch.exp(x - torch.where(top > -math.inf, top, torch.zeros_like(top)))
                e = torch.where(seen, e, torch.zeros_like(e))
                s = e.sum(1, keepdim=True)
                p = e / torch.where(s > 0, s, torch.ones_like(s))
                # a change of the scores by at most d changes a weight by at most exp(2 d) - 1 of itself; the running maximum,
                # the change to base 2 and the exponential add roundings of the score and of the result
                xm = torch.where(seen, x.abs(), torch.zeros_like(x)).amax(1, keepdim=True)
                d = torch.where(seen, dx, torch.zeros_like(dx)).amax(1, keepdim=True) + 8 * f * (xm + 1)
                rel = torch.expm1(2 * d) + (nq + 16) * f * 2
                size = p @ vv[h // G].abs()
                o = p @ vv[h // G]
                out[lo:hi, h] = o
                # the weights rounded to the element type for the second product, its fp32 sum, the output rounded
                tol[lo:hi, h] = size * ((u if q.dtype != torch.float32 else 0.0) + rel + (n + 64) * f) + u * o.abs() + 1e-30
                w += p.sum(0)
                wtol += (p * (rel + (n + 64) * f)).sum(0) + (H * nq + 8) * f * p.sum(0)
        ws.append(w)
        wt.append(wtol)
    return out, tol, ws, wt


def evict(pos, weight, n, keep, sink, recent):
    """Moves [(source slot, destination slot)] of one sequence, plainly."""
    keep = max(0, min(keep, n))
    if keep == n:
        return [], n
    last = max(pos[:n])

    def order(w):
        return (1, 0.0) if w != w else (0, w)

    rank = sorted(range(n), key=lambda j: (pos[j] < sink or pos[j] > last - recent, order(weight[j]), pos[j], j))
    gone = set(rank[:n - keep])
    holes = [j for j in range(keep) if j in gone]
    movers = [j for j in range(keep, n) if j not in gone]
    assert len(holes) == len(movers)
    return list(zip(movers, holes)), keep
