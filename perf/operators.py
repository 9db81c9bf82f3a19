"""Attention over a cache in 8 bits, as cases that can be timed and compared.

A case is a dict of plain values.  `kind` names the operator:

    append   Context.kv_append    new keys and values into the cache: open blocks in 16 bits, full ones in 8 with a scale
    attend   Context.kv_attend    attention over the whole cache: single tokens, a few, prompts (causal)
    sparse   Context.kv_select and Context.kv_attend over what it selected: w blocks of 64 tokens for each query token
    evict    Context.kv_evict by the weight that every block has had so far, then Context.kv_attend over what stays,
             with the weight of this step added

B sequences, n query (or new) tokens each, L tokens in the longest sequence's cache, H key/value heads of D dimensions,
g query heads to each of them.  `ragged`: the sequences differ in length and in the number of their query tokens.

The cache is what a program holds between calls: pages of 64 tokens of one head (codes and a power of two as scale, for
keys and for values; the smallest and largest code of every dimension of the keys), a table of pages per sequence and
head, the open block's tokens in 16 bits.  Keys follow topics, one to a block, and queries ask for topics, so that a few
blocks hold most of a query's weight; the pages lie in random order.
"""
import math

import torch

own = False

BLOCK = 64
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # one step of a served batch: one token of every sequence goes into its open block, one in 64 fills it
        dict(name="append_step", kind="append", dtype="bf16", B=64, n=1, L=4000, H=8, g=4, D=128, ragged=True),
        # four prompts of 8192 tokens
        dict(name="append_prompts", kind="append", dtype="bf16", B=4, n=8192, L=0, H=8, g=4, D=128, ragged=False),
        # one user's step: latency
        dict(name="attend_one", kind="attend", dtype="bf16", B=1, n=1, L=1000, H=8, g=4, D=128, ragged=False),
        # one step of a served batch, lengths from 129 to 8192
        dict(name="attend_batch", kind="attend", dtype="bf16", B=64, n=1, L=8192, H=8, g=4, D=128, ragged=True),
        # a few long documents, a draft of four tokens to be checked, sixteen rows to a head
        dict(name="attend_long", kind="attend", dtype="fp16", B=4, n=4, L=100_000, H=8, g=4, D=128, ragged=False),
        # two prompts, causal
        dict(name="attend_prompts", kind="attend", dtype="bf16", B=2, n=4096, L=4096, H=8, g=4, D=128, ragged=False),
        # the next pieces of three prompts over what is cached already; no size is a multiple of anything
        dict(name="attend_ragged", kind="attend", dtype="fp16", B=3, n=1000, L=10_001, H=4, g=5, D=96, ragged=True),
        # a step of a served batch, 16 blocks of 512
        dict(name="sparse_batch", kind="sparse", dtype="bf16", B=32, n=1, L=32_768, H=8, g=4, D=128, ragged=True, w=16, sink=1, recent=1),
        # a million tokens, 100 blocks of them
        dict(name="sparse_million", kind="sparse", dtype="bf16", B=1, n=1, L=1_000_000, H=8, g=8, D=128, ragged=False, w=100, sink=1, recent=4),
        # a piece of a prompt over a long past, every token with its own blocks
        dict(name="sparse_prompt", kind="sparse", dtype="bf16", B=1, n=1000, L=16_384, H=8, g=4, D=128, ragged=False, w=16, sink=1, recent=2),
        # a step at which caches of up to 8192 tokens are cut to 4096
        dict(name="evict_step", kind="evict", dtype="bf16", B=16, n=1, L=8192, H=8, g=4, D=128, ragged=True, budget=64, sink=1, recent=4),
        # a piece of a prompt after the past was cut to 100 blocks
        dict(name="evict_prompt", kind="evict", dtype="fp16", B=2, n=256, L=20_000, H=8, g=3, D=64, ragged=False, budget=100, sink=2, recent=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0), _cost(c))
    while True:
        kind = rng.choice(["append", "attend", "attend", "attend", "sparse", "sparse", "evict"])
        D = rng.choice([64, 96, 128, 128])
        g = rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8, 8, 12, 16])
        c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "fp16"]), B=_log(rng, 1, 64), n=1, L=_log(rng, 1, 200_000), H=rng.choice([1, 2, 4, 5, 8, 8]), g=g, D=D, ragged=rng.random() < 0.5)
        if kind == "append":
            c["n"] = _log(rng, 1, 8192)
        elif rng.random() < 0.5:
            c["n"] = _log(rng, 2, 4096 if kind == "attend" else 1000)
        if kind == "sparse":
            c["w"] = _log(rng, 4, 100)
            c["sink"], c["recent"] = rng.choice([0, 1, 2]), rng.choice([0, 1, 2])
            if c["n"] > 1 and c["B"] * c["n"] * c["H"] * c["w"] > 1000 * 8 * 17:  # what the plain form gathers for each token
                continue
        if kind == "evict":
            c["budget"] = _log(rng, 8, 200)
            c["sink"], c["recent"] = rng.choice([0, 1, 2]), rng.choice([1, 2, 4])
            if c["budget"] < c["sink"] + c["recent"] + c["n"] // BLOCK + 1:
                continue
        if kind != "append" and c["L"] < c["n"]:
            continue
        rows = c["B"] * c["H"] * g * c["n"]
        if kind != "append" and kind != "sparse" and rows * c["L"] > 2 * 32 * 4096 * 4096:  # the plain form's logits
            continue
        if c["B"] * c["H"] * (c["L"] + c["n"]) > 8_500_000 or _cost(c) > most[kind]:
            continue
        return c


def _counts(case):
    """Query (or new) tokens of every sequence: all n, or down to a third of them."""
    B, n = case["B"], case["n"]
    return [n - (b * 7919) % max(1, 2 * n // 3) if case["ragged"] and n > 1 else n for b in range(B)]


def _lens(case):
    """Tokens in every sequence's cache: before the call for append, with the query tokens for the others."""
    B, L, counts = case["B"], case["L"], _counts(case)
    lens = [L * (b + 1) // B - (b * 13) % 29 if case["ragged"] else L for b in range(B)]
    if case["kind"] == "append":
        # prompts start empty, their later pieces at a block's start; steps and short pieces anywhere
        return [max(0, x) // (BLOCK if case["n"] > BLOCK else 1) * (BLOCK if case["n"] > BLOCK else 1) for x in lens]
    return [max(1, c, x) for x, c in zip(lens, counts)]


def _kept(case):
    """Tokens that stay after the eviction of an evict case."""
    return [min(x // BLOCK, case["budget"]) * BLOCK + x % BLOCK for x in _evict_lens(case)]


def _evict_lens(case):
    """Tokens that an evict case's cache holds: no query token lies in a block that can go."""
    least = (case["n"] // BLOCK + 2 + case["recent"] + case["sink"]) * BLOCK
    return [max(x, least) if x // BLOCK > case["budget"] else x for x in _lens(case)]


def _recent(case):
    """The last blocks that stay: those of the query tokens too."""
    return case["recent"] + case["n"] // BLOCK + 1


def work(case):
    H, g, D, n = case["H"], case["g"], case["D"], case["n"]
    lens, counts = _lens(case), _counts(case)
    token = 2 * D + 8 / BLOCK  # bytes of a cached token of one head
    if case["kind"] == "append":
        moved = 0
        for x, c in zip(lens, counts):
            full = (x % BLOCK + c) // BLOCK
            left = (x % BLOCK + c) % BLOCK if full else c
            old = x % BLOCK if full else 0  # what the open block held when it fills up
            moved += c * 4 * D + old * 4 * D + full * (BLOCK * token + 2 * D) + left * 4 * D
        return {"bytes": H * moved, "flops": H * sum(counts) * 2 * D * 3}
    rows = sum(counts) * H * g
    inout = rows * D * 4 + rows * 4
    if case["kind"] == "evict":
        lens = _kept(case)
        inout += sum(x // BLOCK for x in _evict_lens(case)) * H * 16
    if case["kind"] == "sparse":
        w, seen, flops, cheap = case["w"], 0, 0, 0
        for x, c in zip(lens, counts):
            for i in (range(c) if c <= 64 else [c // 2] * c):
                vis = x - c + i + 1
                t = min(w, vis // BLOCK) * BLOCK + vis % BLOCK
                seen += t
                flops += t * 4 * D
                cheap += vis // BLOCK
        bounds = sum(x // BLOCK for x in lens) * H * (2 * D + 4)
        # a token's blocks are its own, but no block need come from memory more than once
        return {"bytes": inout + bounds + min(seen, sum(lens)) * H * token, "flops": flops * H * g + cheap * H * g * 4 * D}
    pairs = sum(c * x - c * (c - 1) // 2 for x, c in zip(lens, counts))
    return {"bytes": inout + sum(lens) * H * token, "flops": pairs * H * g * 4 * D}


# ---- inputs


def _seal(x):
    """Blocks [..., 64, D] in float32 as codes and scales: the smallest power of two that leaves every value within 448."""
    m, e = torch.frexp(x.abs().amax((-1, -2)))
    e = (e - torch.where(m <= 0.875, 9, 8)).clamp(-126, 119)
    scale = torch.ldexp(torch.ones_like(m), torch.where(m > 0, e, 0))
    return (x / scale[..., None, None]).to(torch.float8_e4m3fn), scale


def _cache(case, lens, room, rand):
    """A cache with `lens` tokens and room for `room` more in every sequence; the topics of its keys."""
    B, H, D, T = case["B"], case["H"], case["D"], TYPES[case["dtype"]]
    dev = "cuda"
    full = [x // BLOCK for x in lens]
    blocks = max((x + r) // BLOCK for x, r in zip(lens, room)) + 1
    need = [(x + r) // BLOCK for x, r in zip(lens, room)]
    pages = max(1, H * sum(need) + 3)
    order = torch.randperm(pages, generator=rand, device=dev).to(torch.int32)
    c = dict(k=torch.zeros(pages, BLOCK, D, device=dev, dtype=torch.float8_e4m3fn), v=torch.zeros(pages, D, BLOCK, device=dev, dtype=torch.float8_e4m3fn),
             scales=torch.ones(pages, 2, device=dev), bounds=torch.zeros(pages, 2, D, device=dev, dtype=torch.float8_e4m3fn),
             tail_k=torch.randn(B, H, 2, BLOCK, D, generator=rand, device=dev).to(T), tail_v=torch.randn(B, H, 2, D, BLOCK, generator=rand, device=dev).to(T),
             table=torch.full((B, H, blocks), -1, device=dev, dtype=torch.int32), lens=torch.tensor(lens, device=dev, dtype=torch.int32),
             evicted=torch.randint(0, 2, (B,), generator=rand, device=dev, dtype=torch.int32))
    topics = torch.randn(B, H, 32, D, generator=rand, device=dev)
    at = 0
    for b in range(B):
        if need[b]:
            c["table"][b, :, : need[b]] = order[at : at + H * need[b]].view(H, need[b])
        at += H * need[b]
        for h0 in range(0, H if full[b] else 0, 2):  # two heads at a time: a million tokens of all of them take much room
            hs = slice(h0, min(H, h0 + 2))
            of = torch.randint(0, 32, (topics[b, hs].shape[0], full[b], 1), generator=rand, device=dev).expand(-1, -1, D)
            x = 0.8 * topics[b, hs].gather(1, of)[:, :, None] + torch.randn(of.shape[0], full[b], BLOCK, D, generator=rand, device=dev)
            page = c["table"][b, hs, : full[b]].long()
            codes, scale = _seal(x.to(T).float())
            c["k"][page], c["scales"][page, 0] = codes, scale
            c["bounds"][page, 0], c["bounds"][page, 1] = codes.float().amin(-2).to(torch.float8_e4m3fn), codes.float().amax(-2).to(torch.float8_e4m3fn)
            x = torch.randn(x.shape, generator=rand, device=dev) * (0.5 + torch.rand(x.shape[0], 1, 1, D, generator=rand, device=dev))
            codes, scale = _seal(x.to(T).float())
            c["v"][page], c["scales"][page, 1] = codes.transpose(-1, -2), scale
    return c, topics


def prepare(case, seed):
    rand = torch.Generator(device="cuda")
    rand.manual_seed(int(seed))
    B, n, H, g, D, T = case["B"], case["n"], case["H"], case["g"], case["D"], TYPES[case["dtype"]]
    counts = _counts(case)
    s = dict(case=case, counts=torch.tensor(counts, device="cuda", dtype=torch.int32) if case["ragged"] else None)
    if case["kind"] == "append":
        s["cache"], _ = _cache(case, _lens(case), counts, rand)
        spread = torch.exp(0.5 * torch.randn(2, 1, 1, H, D, generator=rand, device="cuda"))
        s["k"] = (spread[0] * torch.randn(B, n, H, D, generator=rand, device="cuda")).to(T)
        s["v"] = (spread[1] * torch.randn(B, n, H, D, generator=rand, device="cuda")).to(T)
        return s
    lens = _evict_lens(case) if case["kind"] == "evict" else _lens(case)
    s["cache"], topics = _cache(case, lens, [0] * B, rand)
    of = torch.randint(0, 32, (B, H, n, 1), generator=rand, device="cuda").expand(-1, -1, -1, D)
    q = topics.gather(2, of)[:, :, :, None] + torch.randn(B, H, n, g, D, generator=rand, device="cuda")
    s["q"] = q.permute(0, 2, 1, 3, 4).reshape(B, n, H * g, D).to(T)
    if case["kind"] == "evict":
        # what earlier steps have left: a few blocks hold most of it
        s["mass"] = torch.exp(2 * torch.randn(s["cache"]["table"].shape, generator=rand, device="cuda"))
    return s


# ---- the operators


def run(state):
    return _own_run(state) if own else _plain_run(state)


def _own_run(s):
    import paper_1509_05186_amd as etf

    if "context" not in s:
        s["context"] = etf.Context(device=0, stream=torch.cuda.current_stream().cuda_stream)
        s["handle"] = etf.KvCache(**s["cache"])
    case, ctx, cache = s["case"], s["context"], s["handle"]
    if case["kind"] == "append":
        ctx.kv_append(cache, s["k"], s["v"], counts=s["counts"])
        return {x: s["cache"][x] for x in ("k", "v", "scales", "bounds", "tail_k", "tail_v")}
    lse = torch.empty(s["q"].shape[:3], device=s["q"].device)
    if case["kind"] == "attend":
        return {"out": ctx.kv_attend(cache, s["q"], counts=s["counts"], lse=lse), "lse": lse}
    if case["kind"] == "sparse":
        lists = ctx.kv_select(cache, s["q"], case["w"], sink=case["sink"], recent=case["recent"], counts=s["counts"])
        return {"lists": lists, "out": ctx.kv_attend(cache, s["q"], counts=s["counts"], lists=lists, lse=lse), "lse": lse}
    to = cache.fork()
    kept, freed = ctx.kv_evict(cache, s["mass"], case["budget"], sink=case["sink"], recent=_recent(case), to=to)
    mass = torch.empty_like(kept)
    out = ctx.kv_attend(to, s["q"], counts=s["counts"], lse=lse, mass_in=kept, mass_out=mass)
    return {"table": to.table, "lens": to.lens, "evicted": to.evicted, "kept": kept, "freed": freed, "out": out, "lse": lse, "mass": mass}


def _plain_run(s):
    case, c = s["case"], s["cache"]
    if case["kind"] == "append":
        return _plain_append(c, s["k"], s["v"], s["counts"])
    if case["kind"] == "attend":
        out, lse, _ = _plain_attend(c, s["q"], s["counts"])
        return {"out": out, "lse": lse}
    if case["kind"] == "sparse":
        lists = _plain_select(c, s["q"], s["counts"], case["w"], case["sink"], case["recent"])
        out, lse = _plain_listed(c, s["q"], s["counts"], lists)
        return {"lists": lists, "out": out, "lse": lse}
    to, kept, freed = _plain_evict(c, s["mass"], case["budget"], case["sink"], _recent(case))
    out, lse, mass = _plain_attend(to, s["q"], s["counts"], kept)
    return {"table": to["table"], "lens": to["lens"], "evicted": to["evicted"], "kept": kept, "freed": freed, "out": out, "lse": lse, "mass": mass}


def _plain_append(c, k, v, counts):
    B, n, H, D = k.shape
    dev = k.device
    lens = c["lens"].long()
    counts = torch.full_like(lens, n) if counts is None else counts.long()
    batch = torch.arange(B, device=dev)
    first, begin = lens // BLOCK, lens % BLOCK
    blocks = (BLOCK - 1 + n) // BLOCK + 1
    # the open block's tokens, then the new ones, from the open block's start on
    buf = (first + c["evicted"].long()) % 2
    i = torch.arange(n, device=dev)
    to = torch.where(i < counts[:, None], begin[:, None] + i, blocks * BLOCK)
    old = torch.arange(BLOCK, device=dev)
    full = (begin + counts) // BLOCK
    rest = torch.arange(blocks, device=dev)
    sealed = (rest < full[:, None])[:, None].expand(B, H, blocks)
    column = (first[:, None] + rest).clamp_max(c["table"].shape[2] - 1)[:, None].expand(B, H, blocks)
    page = c["table"].long().gather(2, column)[sealed]
    open_buf = (first + full + c["evicted"].long()) % 2
    staged = []
    for new, tail in ((k, c["tail_k"]), (v, c["tail_v"].transpose(-1, -2))):
        x = torch.zeros(B, H, blocks * BLOCK + 1, D, device=dev, dtype=k.dtype)
        x[:, :, :BLOCK] = torch.where((old < begin[:, None])[:, None, :, None], tail[batch, :, buf], x[:, :, :BLOCK])
        x.scatter_(2, to[:, None, :, None].expand(B, H, n, D), new.transpose(1, 2))
        staged.append(x[:, :, : blocks * BLOCK].view(B, H, blocks, BLOCK, D))
    codes, c["scales"][page, 0] = _seal(staged[0].float()[sealed])
    c["k"][page] = codes
    c["bounds"][page, 0], c["bounds"][page, 1] = codes.float().amin(-2).to(codes.dtype), codes.float().amax(-2).to(codes.dtype)
    codes, c["scales"][page, 1] = _seal(staged[1].float()[sealed])
    c["v"][page] = codes.transpose(-1, -2)
    # what is left lies in the block that is open now; the rest of its buffer stays as it was
    at = full.clamp_max(blocks - 1)
    left = ((begin + counts) % BLOCK)[:, None]
    written = ((old < left) & ((old >= begin[:, None]) | (full > 0)[:, None]))[:, None, :, None]
    tail = c["tail_k"][batch, :, open_buf]
    c["tail_k"][batch, :, open_buf] = torch.where(written, staged[0][batch, :, at], tail)
    tail = c["tail_v"][batch, :, open_buf]
    c["tail_v"][batch, :, open_buf] = torch.where(written.transpose(-1, -2), staged[1][batch, :, at].transpose(-1, -2), tail)
    return {x: c[x] for x in ("k", "v", "scales", "bounds", "tail_k", "tail_v")}


def _seen(c, counts, n):
    """Tokens that query token i of sequence b sees: [B, n]."""
    lens = c["lens"].long()
    counts = torch.full_like(lens, n) if counts is None else counts.long()
    i = torch.arange(n, device=lens.device)
    return torch.where(i < counts[:, None], (lens - counts)[:, None] + i + 1, 0).clamp_min(0)


def _open(c):
    """Keys and values of the open blocks, [B, H, 64, D] each, in float32."""
    lens = c["lens"].long()
    batch, buf = torch.arange(len(lens), device=lens.device), (lens // BLOCK + c["evicted"].long()) % 2
    return c["tail_k"][batch, :, buf].float(), c["tail_v"][batch, :, buf].transpose(-1, -2).float()


def _pages(c, page):
    """Keys and values of pages, [..., 64, D] each, in float32."""
    page = page.long().clamp_min(0)
    scale = c["scales"][page]
    return c["k"][page].float() * scale[..., 0, None, None], c["v"][page].transpose(-1, -2).float() * scale[..., 1, None, None]


def _softmax(logits, valid):
    """Weights without their sum, the sum, and its logarithm with the maximum; nothing seen: zeros."""
    logits = logits.masked_fill_(~valid, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = logits.sub_(top.clamp_min(-3e38)).exp_()
    total = p.sum(-1, keepdim=True)
    return p, total, (top + total.log())[..., 0]


def _plain_attend(c, q, counts, mass=None):
    B, n, Hq, D = q.shape
    H, blocks = c["table"].shape[1:]
    g, dev = Hq // H, q.device
    seen, nb = _seen(c, counts, n), c["lens"].long() // BLOCK
    K, V = _pages(c, c["table"])
    tail = _open(c)
    K, V = (torch.cat([x.flatten(2, 3), t], 2) for x, t in zip((K, V), tail))
    t = torch.arange(blocks * BLOCK, device=dev)
    place = torch.cat([torch.where(t < nb[:, None] * BLOCK, t, 1 << 40), nb[:, None] * BLOCK + torch.arange(BLOCK, device=dev)], 1)
    valid = place[:, None] < seen[:, :, None]  # [B, n, tokens]
    rows = q.view(B, n, H, g, D).transpose(1, 2).reshape(B, H, n * g, D).float()
    logits = (rows @ K.transpose(-1, -2)).mul_(1 / math.sqrt(D))
    p, total, lse = _softmax(logits.view(B, H, n, g, -1), valid[:, None, :, None])
    out = (p.view(B, H, n * g, -1) @ V).view(B, H, n, g, D) / total.clamp_min(1e-37)
    if mass is not None:
        p /= total.clamp_min(1e-37)
        per = p.sum((2, 3)).view(B, H, blocks + 1, BLOCK).sum(-1)
        mass = mass.clone()
        mass += per[..., :blocks]
        mass.scatter_add_(2, nb.clamp_max(blocks - 1)[:, None, None].expand(B, H, 1), per[..., blocks:] * (nb < blocks)[:, None, None])
    return out.transpose(1, 2).reshape(B, n, Hq, D).to(q.dtype), lse.transpose(1, 2).reshape(B, n, Hq), mass


def _plain_select(c, q, counts, w, sink, recent):
    B, n, Hq, D = q.shape
    H, blocks = c["table"].shape[1:]
    g = Hq // H
    page = c["table"].long().clamp_min(0)
    lo, hi = (c["bounds"][page][..., x, :].double().transpose(-1, -2) for x in (0, 1))
    rows = q.view(B, n, H, g, D).transpose(1, 2).reshape(B, H, n * g, D).double()
    score = rows.clamp_min(0) @ hi + rows.clamp_max(0) @ lo
    score = (score * c["scales"][page][:, :, None, :, 0].double()).view(B, H, n, g, blocks).amax(3)
    whole = (_seen(c, counts, n) // BLOCK)[:, None, :, None]
    j = torch.arange(blocks, device=q.device)
    score = torch.where((j < sink) | (j >= whole - recent), math.inf, score)
    score = torch.where(j < whole, score, -math.inf)
    if w > blocks:
        score = torch.nn.functional.pad(score, (0, w - blocks), value=-math.inf)
    value, index = torch.sort(score, dim=-1, descending=True, stable=True)
    index = torch.where(value[..., :w] > -math.inf, index[..., :w], 1 << 40).sort(-1)[0]
    return torch.where(index < 1 << 40, index, -1).to(torch.int32).transpose(1, 2).contiguous()


def _plain_listed(c, q, counts, lists):
    B, n, Hq, D = q.shape
    H, blocks = c["table"].shape[1:]
    g, dev = Hq // H, q.device
    seen, nb = _seen(c, counts, n), c["lens"].long() // BLOCK
    # the listed blocks, and the one that the token sees a part of
    part = (seen // BLOCK)[:, :, None, None].expand(B, n, H, 1)
    index = torch.cat([lists.long(), part], -1)
    page = c["table"].long()[:, None].expand(B, n, H, blocks).gather(3, index.clamp(0, blocks - 1))
    K, V = _pages(c, page)
    tail, is_open = _open(c), (part[..., 0] == nb[:, None, None])[..., None, None]
    for x, t in zip((K, V), tail):
        x[:, :, :, -1] = torch.where(is_open, t[:, None], x[:, :, :, -1])
    place = index[..., None] * BLOCK + torch.arange(BLOCK, device=dev)
    valid = ((place < seen[:, :, None, None, None]) & (index >= 0)[..., None]).flatten(3)
    logits = (q.view(B, n, H, g, D).float() @ K.flatten(3, 4).transpose(-1, -2)).mul_(1 / math.sqrt(D))
    p, total, lse = _softmax(logits, valid[:, :, :, None])
    out = (p @ V.flatten(3, 4)) / total.clamp_min(1e-37)
    return out.view(B, n, Hq, D).to(q.dtype), lse.reshape(B, n, Hq)


def _plain_evict(c, mass, budget, sink, recent):
    B, H, blocks = c["table"].shape
    lens, j = c["lens"].long(), torch.arange(blocks, device=mass.device)
    nb = (lens // BLOCK)[:, None, None]
    cut = (nb > budget).expand(B, H, 1)
    rank = torch.where((j < sink) | (j >= nb - recent), math.inf, mass.double())
    rank = torch.where(j < nb, rank, -math.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True)[1]
    place = torch.empty_like(order).scatter_(2, order, j.expand(B, H, blocks))
    stays = torch.where(cut, place < budget, j < nb)
    goes = (j < nb) & ~stays
    stays = stays | (j == nb)  # the open block's weight moves along
    # the blocks that stay, then those that go, in their order
    at = torch.where(stays, 0, torch.where(goes, 1, 2)).sort(dim=-1, stable=True)[1]
    left = stays.sum(-1, keepdim=True)
    kept = torch.where(j < left, mass.gather(2, at), 0)
    table = torch.where(j < torch.minimum(nb, torch.full_like(nb, budget)), c["table"].gather(2, at), -1)
    at = torch.where(goes, 0, 1).sort(dim=-1, stable=True)[1]
    freed = torch.where(j < goes.sum(-1, keepdim=True), c["table"].gather(2, at), -1)
    removed = (lens // BLOCK - budget).clamp_min(0)
    to = dict(c, table=table, lens=(lens - removed * BLOCK).to(torch.int32), evicted=(c["evicted"] + removed).to(torch.int32))
    return to, kept, freed


# ---- the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    c, kind = s["cache"], case["kind"]
    lens, evicted = c["lens"].tolist(), c["evicted"].tolist()
    counts = [case["n"]] * case["B"] if s["counts"] is None else s["counts"].tolist()
    if kind == "append":
        return _exact_append(case, s, lens, evicted, counts)
    if 4.0 * case["B"] * case["n"] * max(lens) * case["H"] * case["g"] * case["D"] > 4e12:
        return None
    if kind == "attend":
        out, lse, _ = _exact_attend(case, s, c["table"], lens, evicted, counts)
        return {"out": out, "lse": lse}
    if kind == "sparse":
        out, lse, _ = _exact_attend(case, s, c["table"], lens, evicted, counts, choose=True)
        return {"lists": None, "out": out, "lse": lse}
    B, H, blocks = c["table"].shape
    table, kept, after = c["table"].clone(), torch.zeros_like(s["mass"], dtype=torch.float64), []
    weight = s["mass"].cpu().tolist()
    for b in range(B):
        nb = lens[b] // BLOCK
        last = case["recent"] + case["n"] // BLOCK + 1
        for h in range(H):
            stay = set(range(nb))
            if nb > case["budget"]:
                middle = sorted(range(case["sink"], nb - last), key=lambda j: (-weight[b][h][j], j))
                stay = set(range(case["sink"])) | set(range(nb - last, nb)) | set(middle[: case["budget"] - case["sink"] - last])
            stay = torch.tensor(sorted(stay), device=table.device, dtype=torch.long)
            table[b, h, : len(stay)] = c["table"][b, h][stay]
            also = torch.cat([stay, stay.new_tensor([nb])]) if nb < blocks else stay
            kept[b, h, : len(also)] = s["mass"][b, h][also].double()
        after.append(max(0, nb - case["budget"]))
    lens = [x - r * BLOCK for x, r in zip(lens, after)]
    evicted = [x + r for x, r in zip(evicted, after)]
    out, lse, added = _exact_attend(case, s, table, lens, evicted, counts)
    return {"table": None, "lens": None, "evicted": None, "kept": kept, "freed": None, "out": out, "lse": lse, "mass": kept + added}


def _exact_round(x):
    """x [64, D] in float64 as e4m3 values (float64) and their scale: three bits after the leading one, steps of 2^-9 at least."""
    most = float(x.abs().max())
    e = -126
    if most == 0.0:
        e = 0
    else:
        e = max(e, math.frexp(most)[1] - 10)
        while most > 448.0 * 2.0**e:
            e += 1
    y = x / 2.0**e
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0**-6))) - 3)
    return torch.round(y / step) * step, 2.0**e


def _exact_append(case, s, lens, evicted, counts):
    if case["B"] * case["H"] * (case["n"] + BLOCK) > 400_000:
        return None
    c = s["cache"]
    got = {x: c[x].double() for x in ("k", "v", "scales", "bounds", "tail_k", "tail_v")}
    table = c["table"].tolist()
    for b in range(case["B"]):
        first, begin = lens[b] // BLOCK, lens[b] % BLOCK
        old, now = (first + evicted[b]) % 2, ((lens[b] + counts[b]) // BLOCK + evicted[b]) % 2
        for h in range(case["H"]):
            k = torch.cat([c["tail_k"][b, h, old, :begin], s["k"][b, : counts[b], h]]).double()
            v = torch.cat([c["tail_v"][b, h, old, :, :begin].T, s["v"][b, : counts[b], h]]).double()
            whole = len(k) // BLOCK
            for j in range(whole):
                page = table[b][h][first + j]
                x, scale = _exact_round(k[j * BLOCK : (j + 1) * BLOCK])
                got["k"][page], got["scales"][page, 0] = x, scale
                got["bounds"][page, 0], got["bounds"][page, 1] = x.min(0)[0], x.max(0)[0]
                x, got["scales"][page, 1] = _exact_round(v[j * BLOCK : (j + 1) * BLOCK])
                got["v"][page] = x.T
            left = len(k) - whole * BLOCK
            got["tail_k"][b, h, now, :left] = k[whole * BLOCK :]
            got["tail_v"][b, h, now, :, :left] = v[whole * BLOCK :].T
    return got


def _exact_attend(case, s, table, lens, evicted, counts, choose=False):
    c, n, g, D = s["cache"], case["n"], case["g"], case["D"]
    B, H, blocks = table.shape
    dev = table.device
    out = torch.zeros(B, n, H, g, D, device=dev, dtype=torch.float64)
    lse = torch.full((B, n, H, g), -math.inf, device=dev, dtype=torch.float64)
    mass = torch.zeros(B, H, blocks, device=dev, dtype=torch.float64)
    q = s["q"].view(B, n, H, g, D)
    for b in range(B):
        nb, left, m = lens[b] // BLOCK, lens[b] % BLOCK, counts[b]
        buf = (nb + evicted[b]) % 2
        vis = torch.arange(m, device=dev) + (lens[b] - m + 1)
        t = torch.arange(lens[b], device=dev)
        for h in range(H):
            page = table[b, h, :nb].long()
            scale = c["scales"][page].double()
            k = (c["k"][page].double() * scale[:, 0].view(-1, 1, 1)).reshape(-1, D)
            v = (c["v"][page].double() * scale[:, 1].view(-1, 1, 1)).permute(0, 2, 1).reshape(-1, D)
            k = torch.cat([k, c["tail_k"][b, h, buf, :left].double()])
            v = torch.cat([v, c["tail_v"][b, h, buf, :, :left].double().T])
            at = max(1, min(m, 300_000_000 // (g * max(lens[b], 1 + nb * D if choose else 1))))
            for i in range(0, m, at):
                x = q[b, i : i + at, h][: m - i].double()  # [tokens, g, D]
                see = t < vis[i : i + at, None]
                if choose:
                    pick = _exact_choice(case, x, c["bounds"][page].double(), scale[:, 0], vis[i : i + at] // BLOCK)
                    pick = torch.cat([pick, pick.new_zeros(len(pick), 1)], 1)
                    pick.scatter_(1, (vis[i : i + at] // BLOCK)[:, None], True)
                    see = see & pick.gather(1, (t // BLOCK).expand(len(x), -1))
                z = torch.einsum("igd,td->igt", x, k) / math.sqrt(D)
                z = torch.where(see[:, None], z, -math.inf)
                top = torch.logsumexp(z, -1)
                p = torch.exp(z - top[..., None])
                out[b, i : i + len(x), h] = torch.einsum("igt,td->igd", p, v)
                lse[b, i : i + len(x), h] = top
                each = torch.nn.functional.pad(p.sum((0, 1)), (0, (nb + 1) * BLOCK - lens[b])).view(nb + 1, BLOCK).sum(1)
                mass[b, h, : nb + 1] += each[: blocks]
    return out.view(B, n, H * g, D), lse.view(B, n, H * g), mass


def _exact_choice(case, x, bounds, scale, whole):
    """Which blocks every token takes: [tokens, blocks] truth values."""
    nb = len(bounds)
    j = torch.arange(nb, device=x.device)
    best = torch.full((len(x), nb), -math.inf, device=x.device, dtype=torch.float64)
    for r in range(x.shape[1]):
        bound = torch.maximum(x[:, r, None] * bounds[:, 0], x[:, r, None] * bounds[:, 1]).sum(-1) * scale
        best = torch.maximum(best, bound)
    forced = (j < case["sink"]) | (j >= whole[:, None] - case["recent"])
    best = torch.where(forced, math.inf, best)
    best = torch.where(j < whole[:, None], best, -math.inf)
    order = torch.argsort(-best, dim=-1, stable=True)[:, : case["w"]]
    picked = torch.zeros(len(x), nb, device=x.device, dtype=torch.bool).scatter_(1, order, True)
    return picked & (best > -math.inf)
