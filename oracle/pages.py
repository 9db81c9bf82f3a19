"""Pages of the attention cache, entry by entry: what etf_kv_take, _fork, _free and _compact have to give.

A cache is a dict of CPU tensors as in oracle/kvcache.py, refs an int32 tensor.  Plain loops; nothing here is shared with the library.
"""
import torch

from . import kvcache

BLOCK = 64


def _len(c, b):
    return min(max(int(c["lens"][b]), 0), c["table"].shape[2] * BLOCK + BLOCK - 1)


def count(c):
    """refs as the table has them."""
    refs, pages = torch.zeros(c["k"].shape[0], dtype=torch.int32), c["k"].shape[0]
    for p in c["table"].flatten().tolist():
        if 0 <= p < pages:
            refs[p] += 1
    return refs


def take(c, refs, n, counts=None):
    """(table, refs, missing) after pages were given to the blocks that an append completes."""
    B, H, blocks = c["table"].shape
    pages = len(refs)
    table, after = c["table"].clone(), refs.clone()
    free = [p for p in range(pages) if refs[p] <= 0]
    want = []
    for b in range(B):
        k = n if counts is None else min(max(int(counts[b]), 0), n)
        for h in range(H):
            for j in range(_len(c, b) // BLOCK, min((_len(c, b) + k) // BLOCK, blocks)):
                p = int(table[b, h, j])
                if not (0 <= p < pages and refs[p] == 1):
                    want.append((b, h, j, p))
    if len(want) > len(free):
        return table, after, len(want) - len(free)
    for (b, h, j, p), new in zip(want, free):
        if 0 <= p < pages and refs[p] > 1:
            after[p] -= 1
        table[b, h, j] = new
        after[new] = 1
    return table, after, 0


def fork(c, refs, source, keep=None):
    """The cache and refs after every sequence became a copy."""
    B, H, blocks = c["table"].shape
    pages = len(refs)
    new = {name: t.clone() for name, t in c.items() if name in ("table", "lens", "evicted", "tail_k", "tail_v")}
    after = refs.clone()
    for b in range(B):
        s = int(source[b])
        known = 0 <= s < B
        tokens = _len(c, s) if known else 0
        if known and keep is not None and int(keep[b]) < tokens:
            tokens = max(0, int(keep[b])) // BLOCK * BLOCK
        if s == b and tokens == _len(c, b):
            continue
        for h in range(H):
            for j in range(blocks):
                was, now = int(c["table"][b, h, j]), int(c["table"][s, h, j]) if j < tokens // BLOCK else -1
                new["table"][b, h, j] = now
                if 0 <= was < pages:
                    after[was] -= 1
                if 0 <= now < pages:
                    after[now] += 1
            if known and s != b:
                half, left = (tokens // BLOCK + int(c["evicted"][s])) % 2, tokens % BLOCK
                new["tail_k"][b, h, half, :left] = c["tail_k"][s, h, half, :left]
                new["tail_v"][b, h, half, :, :left] = c["tail_v"][s, h, half, :, :left]
        new["lens"][b], new["evicted"][b] = tokens, c["evicted"][s] if known else 0
    return dict(c, **new), after


def free(refs, pages):
    after = refs.clone()
    for p in pages.flatten().tolist():
        if 0 <= p < len(refs) and after[p] > 0:
            after[p] -= 1
    return after


def evict(c, mass, budget, sink, recent):
    """(table, lens, evicted, mass, freed) after an eviction that keeps the entries past the full blocks."""
    table, lens, evicted, kept, freed = kvcache.evict(c, mass, budget, sink, recent)
    blocks = table.shape[2]
    for b in range(table.shape[0]):
        full, stay = _len(c, b) // BLOCK, min(_len(c, b) // BLOCK, budget)
        for h in range(table.shape[1]):
            for j in range(full, blocks):
                table[b, h, stay + j - full] = c["table"][b, h, j]
    return table, lens, evicted, kept, freed


def compact(c, refs):
    """(cache, refs, used): the i-th free page below `used` takes the used page that has i used ones behind it."""
    pages = len(refs)
    taken = [p for p in range(pages) if refs[p] > 0]
    used = len(taken)
    holes = [p for p in range(used) if refs[p] <= 0]
    movers = [p for p in reversed(taken) if p >= used]
    to = dict(zip(movers, holes))
    new = {name: c[name].clone() for name in ("k", "v", "scales", "bounds", "table")}
    after = torch.where(refs > 0, refs, 0)
    for old, p in to.items():
        for name in ("k", "v", "scales", "bounds"):
            new[name][p] = c[name][old]
        after[p], after[old] = refs[old], 0
    for i, p in enumerate(c["table"].flatten().tolist()):
        if p in to:
            new["table"].view(-1)[i] = to[p]
    return dict(c, **new), after, used
