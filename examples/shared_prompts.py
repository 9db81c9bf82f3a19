#!/usr/bin/env python3
"""A served attention layer: requests that begin with the same prompt share its pages, and the pool holds what is needed and no more.

    prompt_attend      the shared prompt's attention, in 16 bits, once for all of them
    kv_take            pages for the blocks that come
    kv_append_packed   the prompts' keys and values into the cache
    kv_fork            every request begins as a copy of the shared prompt: whole blocks are shared, the open block is its own;
                       a request that is done is emptied, and another takes its place
    kv_append, kv_attend   the attention of every request's own part over the cache; single tokens
    kv_compact         the pages in use to the front of the pool, once many requests have left

Keys, values and queries are random.  Prints tokens a second, pages with and without sharing, and the largest difference of the last step's attention
from the same attention over the cache's contents in float64.

    python examples/shared_prompts.py --batch 32 --shared 4000 --own 300 --tokens 256
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_1509_05186_amd as etf
from bounded_cache import exact

BLOCK = etf.ETF_KV_BLOCK


def main(argv=None):
    arg = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("batch", 32), ("heads", 8), ("group", 4), ("head-dim", 128), ("shared", 4000), ("own", 300), ("tokens", 256)):
        arg.add_argument("--" + name, type=int, default=value)
    o = arg.parse_args(argv)
    B, H, D, Hq = o.batch, o.heads, o.head_dim, o.heads * o.group
    rand = torch.Generator(device="cuda").manual_seed(1)
    made = lambda *shape: torch.randn(shape, generator=rand, device="cuda").bfloat16()  # noqa: E731
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731

    most = o.shared + o.own + o.tokens
    # a page for every block of the shared prompt, and for what each request adds
    pages = H * (o.shared // BLOCK + B * ((o.own + o.tokens) // BLOCK + 2))
    cache = etf.KvCache.alloc(B, H, D, most, pages=pages)
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    ctx = etf.Context(device=torch.cuda.current_device(), stream=torch.cuda.current_stream().cuda_stream)

    def take(n, counts=None):
        missing = ctx.kv_take(cache, refs, n, counts=counts)
        if int(missing):
            raise RuntimeError("%d pages are lacking" % int(missing))

    torch.cuda.synchronize()
    start = time.perf_counter()
    # the shared prompt is sequence 0's; the others have no tokens yet
    counts = ints([o.shared] + [0] * (B - 1))
    starts = ints([0] + [o.shared] * B)
    q, k, v = made(o.shared, Hq, D), made(o.shared, H, D), made(o.shared, H, D)
    ctx.prompt_attend(q, k, v, starts)
    take(o.shared, counts)
    ctx.kv_append_packed(cache, k, v, starts)
    cache.lens += counts
    # all of them begin with its whole blocks
    whole = o.shared // BLOCK * BLOCK
    ctx.kv_fork(cache, refs, ints([0] * B), keep=ints([whole] * B))
    # every request's own part, of another length each, packed
    lens = [max(1, o.own - b * 37 % o.own) for b in range(B)]
    starts = ints([0] + lens).cumsum(0).to(torch.int32)
    counts = ints(lens)
    k, v = made(sum(lens), H, D), made(sum(lens), H, D)
    take(max(lens), counts)
    ctx.kv_append_packed(cache, k, v, starts)
    cache.lens += counts
    ctx.kv_attend(cache, made(B, max(lens), Hq, D), counts=counts)
    torch.cuda.synchronize()
    prompts = time.perf_counter() - start
    start = time.perf_counter()
    for i in range(o.tokens):
        if i % BLOCK == 0:
            take(min(BLOCK, o.tokens - i))    # for the next steps at once: a wait for the host in 64
        q, k, v = made(B, 1, Hq, D), made(B, 1, H, D), made(B, 1, H, D)
        ctx.kv_append(cache, k, v)
        cache.lens += 1
        out = ctx.kv_attend(cache, q)
    torch.cuda.synchronize()
    decode = time.perf_counter() - start
    alone = int(sum(int(x) // BLOCK for x in cache.lens.tolist())) * H
    held = int((refs > 0).sum())
    off = float((out.double() - exact(cache, q)).abs().max()) if o.tokens else 0.0
    # every second request is done: the pages that only it had are free
    ctx.kv_fork(cache, refs, ints([b if b % 2 == 0 else -1 for b in range(B)]))
    used = int(ctx.kv_compact(cache, refs))
    out = ctx.kv_attend(cache, q) if o.tokens else None
    print("prompts %.0f tokens/s, single tokens %.0f tokens/s, %d pages where %d would be without sharing, %d after every second request has left; largest difference %.2g"
          % ((o.shared + sum(lens)) / prompts, B * o.tokens / max(decode, 1e-9), held, alone, used, off))
    return cache, refs, used, off


if __name__ == "__main__":
    main()
