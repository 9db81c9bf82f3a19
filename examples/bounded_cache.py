#!/usr/bin/env python3
"""A served attention layer whose cache stays bounded: prompts longer than the cache in pieces, then single tokens.

Every piece and every token goes through the calls in the order in which a server makes them:

    kv_append   the new tokens' keys and values into the cache (open blocks in 16 bits, full ones in 8)
    kv_attend   their attention, which also adds up the weight that every block has had; between evictions, single tokens with
                --w look at the w blocks of kv_select only
    kv_evict    down to --budget blocks of 64 tokens a head by that weight; the pages that come free serve the next blocks

Keys, values and queries are random with a topic to each stretch of tokens.  Prints tokens a second and the largest difference of
the last step's attention from the same attention over the cache's contents in float64.

    python examples/bounded_cache.py --batch 8 --prompt 10000 --tokens 512 --budget 64 --w 16
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_1509_05186_amd as etf

BLOCK = etf.ETF_KV_BLOCK


class BoundedCache:
    """An attention cache that holds `budget` full blocks a head and what comes between two evictions."""

    def __init__(self, batch, heads, head_dim, budget, piece, sink=1, recent=2, device="cuda"):
        self.cache = etf.KvCache.alloc(batch, heads, head_dim, budget * BLOCK + piece + BLOCK, device=device)
        self.mass = torch.zeros(self.cache.table.shape, device=device)
        self.freed = torch.empty_like(self.cache.table)
        self.column = torch.arange(self.cache.max_blocks, device=device)
        self.budget, self.sink, self.recent = budget, sink, recent
        self.ctx = etf.Context(device=torch.cuda.current_device(), stream=torch.cuda.current_stream().cuda_stream)

    def append(self, k, v):
        self.ctx.kv_append(self.cache, k, v)
        self.cache.lens += k.shape[1]

    def attend(self, q):
        return self.ctx.kv_attend(self.cache, q, mass_in=self.mass, mass_out=self.mass)

    def attend_to(self, q, w):
        lists = self.ctx.kv_select(self.cache, q, w, sink=self.sink, recent=self.recent)
        return self.ctx.kv_attend(self.cache, q, lists=lists)

    def evict(self):
        c = self.cache
        before, full = c.table.clone(), (c.lens // BLOCK)[:, None, None]
        self.ctx.kv_evict(c, self.mass, self.budget, sink=self.sink, recent=self.recent, freed=self.freed)
        # every row keeps its pages: those of the blocks that stay, the ones taken out, those that no block has had yet
        stay = full.clamp(max=self.budget)
        freed = self.freed.gather(2, (self.column - stay).clamp(min=0).expand_as(before))
        c.table.copy_(torch.where(self.column < stay, c.table, torch.where(self.column < full, freed, before)))


def exact(cache, q):
    """Attention of single tokens q over what the cache holds, in float64."""
    B, _, Hq, D = q.shape
    H = cache.heads
    out = torch.empty(B, 1, Hq, D, dtype=torch.float64, device=q.device)
    for b in range(B):
        length, evicted = int(cache.lens[b]), int(cache.evicted[b])
        full, left = divmod(length, BLOCK)
        for h in range(H):
            page = cache.table[b, h, :full].long()
            scale = cache.scales[page].double()
            k = (cache.k[page].double() * scale[:, :1, None]).reshape(-1, D)
            v = (cache.v[page].double() * scale[:, 1:, None]).transpose(1, 2).reshape(-1, D)
            half = (full + evicted) % 2
            k = torch.cat([k, cache.tail_k[b, h, half, :left].double()])
            v = torch.cat([v, cache.tail_v[b, h, half, :, :left].T.double()])
            rows = slice(h * (Hq // H), (h + 1) * (Hq // H))
            out[b, 0, rows] = torch.softmax(q[b, 0, rows].double() @ k.T * D ** -0.5, -1) @ v
    return out


def main(argv=None):
    arg = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("batch", 8), ("heads", 8), ("group", 4), ("head-dim", 128), ("prompt", 10000), ("piece", 2048), ("tokens", 512), ("budget", 64), ("w", 16)):
        arg.add_argument("--" + name, type=int, default=value)
    o = arg.parse_args(argv)
    B, H, D = o.batch, o.heads, o.head_dim
    rand = torch.Generator(device="cuda").manual_seed(1)
    topics = torch.randn(16, H, D, generator=rand, device="cuda")

    def made(n, topic):
        k = topics[topic] + torch.randn(B, n, H, D, generator=rand, device="cuda")
        v = torch.randn(B, n, H, D, generator=rand, device="cuda")
        q = topics[topic].repeat_interleave(o.group, 0) + torch.randn(B, n, H * o.group, D, generator=rand, device="cuda")
        return k.bfloat16(), v.bfloat16(), q.bfloat16()

    cache = BoundedCache(B, H, D, o.budget, o.piece)
    torch.cuda.synchronize()
    start = time.perf_counter()
    for at in range(0, o.prompt, o.piece):
        k, v, q = made(min(o.piece, o.prompt - at), at // o.piece % 16)
        cache.append(k, v)
        cache.attend(q)
        cache.evict()
    torch.cuda.synchronize()
    prompt = time.perf_counter() - start
    start = time.perf_counter()
    for i in range(o.tokens):
        k, v, q = made(1, i // 100 % 16)
        cache.append(k, v)
        # a token in eight looks at everything, so that the weights go on telling which blocks are asked for
        out = cache.attend(q) if i % 8 == 0 or not o.w else cache.attend_to(q, o.w)
        if i % BLOCK == BLOCK - 1:
            cache.evict()
    torch.cuda.synchronize()
    decode = time.perf_counter() - start
    out = cache.attend(q)
    off = float((out.double() - exact(cache.cache, q)).abs().max())
    print("prompts %.0f tokens/s, single tokens %.0f tokens/s, cache %d to %d of %d tokens, largest difference %.2g"
          % (B * o.prompt / prompt, B * o.tokens / max(decode, 1e-9), int(cache.cache.lens.min()), int(cache.cache.lens.max()), o.prompt + o.tokens, off))
    return cache, off


if __name__ == "__main__":
    main()
