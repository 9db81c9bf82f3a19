"""Causal attention of packed prompts, row by row in float64: what etf_prompt_attend has to give.  Nothing here is shared with the library."""
import math

import torch


def attend(q, k, v, starts, scale):
    """dict of out, lse (rows of no sequence: not a number) and, for bounds on rounding errors: size = sum p |v|, reach = largest |s|,
    mag = largest sum_d |q_d k_d| scale over what a row sees, seen = how many tokens that is, vmax = largest |v| among them."""
    T, Hq, D = q.shape
    g = Hq // k.shape[1]
    z = lambda *s: torch.full(s, math.nan, dtype=torch.float64)  # noqa: E731
    r = dict(out=z(T, Hq, D), lse=z(T, Hq), size=z(T, Hq, D), reach=z(T, Hq), mag=z(T, Hq), seen=z(T, Hq), vmax=z(T, Hq))
    edges = [min(max(int(x), 0), T) for x in starts]
    for a, e in zip(edges, edges[1:]):
        if e <= a:
            continue
        sees = torch.ones(e - a, e - a).tril().bool()
        for x in range(Hq):
            qq, kk, vv = q[a:e, x].double(), k[a:e, x // g].double(), v[a:e, x // g].double()
            s = (qq @ kk.T * scale).masked_fill(~sees, -math.inf)
            lse = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[:, None])
            r["out"][a:e, x], r["lse"][a:e, x], r["size"][a:e, x] = p @ vv, lse, p @ vv.abs()
            r["reach"][a:e, x] = s.abs().masked_fill(~sees, 0).amax(1)
            r["mag"][a:e, x] = (qq.abs() @ kk.abs().T * scale).masked_fill(~sees, 0).amax(1)
            r["seen"][a:e, x] = torch.arange(1, e - a + 1).double()
            r["vmax"][a:e, x] = vv.abs().amax(1).cummax(0).values
    return r


def attend_rowwise(q, k, v, starts, scale):
    """(out, lse) for inputs that hold what is not finite: each row by itself, over what it sees and nothing else."""
    T, Hq, D = q.shape
    g = Hq // k.shape[1]
    out, lse = torch.full((T, Hq, D), math.nan, dtype=torch.float64), torch.full((T, Hq), math.nan, dtype=torch.float64)
    for a, e in zip(starts, starts[1:]):
        for i in range(a, e):
            for x in range(Hq):
                kk, vv = k[a : i + 1, x // g].double(), v[a : i + 1, x // g].double()
                s = kk @ q[i, x].double() * scale
                lse[i, x] = torch.logsumexp(s, 0)
                p = torch.exp(s - lse[i, x])
                there = p > 0
                out[i, x] = (p[:, None] * vv)[there].sum(0) if there.any() else math.nan
    return out, lse
