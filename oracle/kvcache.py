"""Attention over a cache in 8 bits, token by token in float64: what the device calls etf_kv_* have to give.

A cache is a dict of CPU tensors with the names and shapes of paper_1509_05186_amd.KvCache, codes in float8_e4m3fn.  Plain
loops over sequences and heads; nothing here is shared with the library.
"""
import math

import torch

BLOCK = 64
NAN = float("nan")


def new_cache(batch, heads, dim, blocks, dtype, pages=None, table=None):
    pages = batch * heads * blocks if pages is None else pages
    e4m3 = torch.float8_e4m3fn
    if table is None:
        table = torch.arange(batch * heads * blocks, dtype=torch.int32).view(batch, heads, blocks)
    return dict(k=torch.zeros(pages, BLOCK, dim).to(e4m3), v=torch.zeros(pages, dim, BLOCK).to(e4m3), scales=torch.zeros(pages, 2),
                bounds=torch.zeros(pages, 2, dim).to(e4m3), tail_k=torch.zeros(batch, heads, 2, BLOCK, dim, dtype=dtype),
                tail_v=torch.zeros(batch, heads, 2, dim, BLOCK, dtype=dtype), table=table.to(torch.int32),
                lens=torch.zeros(batch, dtype=torch.int32), evicted=torch.zeros(batch, dtype=torch.int32))


def e4m3(x):
    """x (float64, |x| <= 448) rounded to the nearest e4m3 value, ties to even: steps of 2^(exponent - 3), 2^-9 at least."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def scale_of(amax):
    if amax == 0:
        return 1.0
    e = -126
    while amax > 448.0 * 2.0 ** e and e < 119:
        e += 1
    return 2.0 ** e


def _len(c, b):
    return min(max(int(c["lens"][b]), 0), c["table"].shape[2] * BLOCK + BLOCK - 1)


def _page(c, b, h, j):
    p = int(c["table"][b, h, j]) if 0 <= j < c["table"].shape[2] else -1
    return p if 0 <= p < c["k"].shape[0] else -1


def append(c, k, v, counts=None):
    """Writes k, v [B][n][H][D] after c["lens"], as far as lens can count; lens stays."""
    B, n, H, D = k.shape
    for b in range(B):
        count = n if counts is None else min(max(int(counts[b]), 0), n)
        count = min(count, c["table"].shape[2] * BLOCK + BLOCK - 1 - _len(c, b))
        first, begin = _len(c, b) // BLOCK, _len(c, b) % BLOCK
        for h in range(H):
            old = (first + int(c["evicted"][b])) % 2
            kk = torch.cat([c["tail_k"][b, h, old, :begin], k[b, :count, h]])
            vv = torch.cat([c["tail_v"][b, h, old, :, :begin].T, v[b, :count, h]]).clone()
            bad = ~(torch.isfinite(kk).all(1) & torch.isfinite(vv).all(1))
            kk[bad], vv[bad] = NAN, 0
            whole = len(kk) // BLOCK
            for j in range(whole):
                page = _page(c, b, h, first + j)
                if page < 0:
                    continue
                s = slice(j * BLOCK, (j + 1) * BLOCK)
                x, y, ok = kk[s].double(), vv[s].double(), ~bad[s]
                for at, (z, name) in enumerate(((x, "k"), (y, "v"))):
                    scale = scale_of(float(z[ok].abs().max()) if ok.any() else 0.0)
                    code = torch.where(torch.isfinite(z), e4m3((z / scale).clamp(-448, 448)), z)
                    c["scales"][page, at] = scale
                    c[name][page] = (code if name == "k" else code.T).to(torch.float32).to(torch.float8_e4m3fn)
                    if name == "k":
                        for w, edge in enumerate((code[ok].amin(0), code[ok].amax(0)) if ok.any() else (torch.zeros(D),) * 2):
                            c["bounds"][page, w] = edge.to(torch.float32).to(torch.float8_e4m3fn)
            now, left = (first + whole + int(c["evicted"][b])) % 2, len(kk) - whole * BLOCK
            at = 0 if whole else begin
            c["tail_k"][b, h, now, at:left] = kk[whole * BLOCK + at:]
            c["tail_v"][b, h, now, :, at:left] = vv[whole * BLOCK + at:].T


def tokens(c, b, h):
    """(keys, values, is there) of the tokens of one (sequence, head) in float64."""
    n, D = _len(c, b), c["k"].shape[2]
    nb = n // BLOCK
    ks, vs, there = [torch.zeros(0, D).double()], [torch.zeros(0, D).double()], [torch.zeros(0, dtype=torch.bool)]
    for j in range(nb):
        p = _page(c, b, h, j)
        there.append(torch.full((BLOCK,), p >= 0))
        ks.append(c["k"][p].double() * float(c["scales"][p, 0]) if p >= 0 else torch.zeros(BLOCK, D).double())
        vs.append(c["v"][p].double().T * float(c["scales"][p, 1]) if p >= 0 else torch.zeros(BLOCK, D).double())
    buf = (nb + int(c["evicted"][b])) % 2
    ks.append(c["tail_k"][b, h, buf, : n % BLOCK].double())
    vs.append(c["tail_v"][b, h, buf, :, : n % BLOCK].double().T)
    there.append(torch.ones(n % BLOCK, dtype=torch.bool))
    return torch.cat(ks), torch.cat(vs), torch.cat(there)


def attend(c, q, scale, counts=None, lists=None):
    """dict of out, lse, mass and, for bounds on rounding errors: size = sum p |v|, reach = largest |s|, mag = largest sum_d |q_d k_d| scale
    over what a row sees, seen = how many tokens that is, vmax."""
    B, n, Hq, D = q.shape
    H, blocks = c["table"].shape[1:]
    g = Hq // H
    z = lambda *s: torch.zeros(*s, dtype=torch.float64)  # noqa: E731
    r = dict(out=z(B, n, Hq, D), lse=torch.full((B, n, Hq), -math.inf).double(), mass=z(B, H, blocks), size=z(B, n, Hq, D), reach=z(B, n, Hq),
             mag=z(B, n, Hq), seen=z(B, n, Hq), vmax=z(B, n, Hq))
    for b in range(B):
        count = n if counts is None else min(max(int(counts[b]), 0), n)
        for h in range(H):
            k, v, there = tokens(c, b, h)
            for i in range(count):
                vis = max(0, _len(c, b) - count + i + 1)
                see = there.clone()
                see[vis:] = False
                if lists is not None:
                    whole = vis // BLOCK
                    listed = {int(j) for j in lists[b, i, h] if 0 <= int(j) < whole}
                    for j in range(whole):
                        if j not in listed:
                            see[j * BLOCK : (j + 1) * BLOCK] = False
                if not see.any():
                    continue
                for x in range(h * g, h * g + g):
                    qq = q[b, i, x].double()
                    s = (k[see] @ qq) * scale
                    lse = torch.logsumexp(s, 0)
                    p = torch.exp(s - lse)
                    r["out"][b, i, x], r["lse"][b, i, x] = p @ v[see], lse
                    r["size"][b, i, x], r["reach"][b, i, x] = p @ v[see].abs(), s.abs().max()
                    r["mag"][b, i, x], r["seen"][b, i, x] = (k[see].abs() @ qq.abs()).max() * scale, len(s)
                    r["vmax"][b, i, x] = v[see].abs().max()
                    every = z((blocks + 1) * BLOCK)
                    every[: len(see)][see] = p
                    r["mass"][b, h] += every.view(-1, BLOCK).sum(1)[:blocks]
    return r


def select(c, q, w, sink, recent, counts=None):
    B, n, Hq, D = q.shape
    H, blocks = c["table"].shape[1:]
    g = Hq // H
    lists = torch.full((B, n, H, w), -1, dtype=torch.int32)
    for b in range(B):
        count = n if counts is None else min(max(int(counts[b]), 0), n)
        for i in range(count):
            whole = min(max(0, _len(c, b) - count + i + 1) // BLOCK, blocks)
            for h in range(H):
                ranked = []
                for j in range(whole):
                    p = _page(c, b, h, j)
                    if p < 0:
                        continue
                    lo, hi = c["bounds"][p].double()
                    score = max(float(torch.maximum(x * lo, x * hi).sum()) for x in q[b, i, h * g : h * g + g].double()) * float(c["scales"][p, 0])
                    if j < sink or j >= whole - recent:
                        score = math.inf
                    ranked.append((-score, j))
                got = sorted(j for _, j in sorted(ranked)[:w])
                lists[b, i, h, : len(got)] = torch.tensor(got, dtype=torch.int32)
    return lists


def evict(c, mass, budget, sink, recent):
    """(table, lens, evicted, mass, freed) after the eviction."""
    B, H, blocks = c["table"].shape
    table, freed, out = torch.full_like(c["table"], -1), torch.full_like(c["table"], -1), torch.zeros_like(mass)
    lens, evicted = c["lens"].clone(), c["evicted"].clone()
    for b in range(B):
        n = _len(c, b)
        nb = n // BLOCK
        nb = min(nb, blocks)
        gone = max(0, nb - budget)
        lens[b], evicted[b] = n - gone * BLOCK, evicted[b] + gone
        for h in range(H):
            stay = set(range(nb))
            if gone:
                rank = sorted(range(nb), key=lambda j: (0 if j < sink or j >= nb - recent else 1, math.inf if math.isnan(mass[b, h, j]) else -float(mass[b, h, j]), j))
                stay = set(rank[:budget])
            kept, out_ = sorted(stay), [j for j in range(nb) if j not in stay]
            table[b, h, : len(kept)] = c["table"][b, h, kept]
            out[b, h, : len(kept)] = mass[b, h, kept]
            if nb < blocks:
                out[b, h, len(kept)] = mass[b, h, nb]
            freed[b, h, : len(out_)] = c["table"][b, h, out_]
    return table, lens, evicted, out, freed
