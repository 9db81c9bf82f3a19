"""Packed prompts and the pages of an attention cache, as cases that can be timed and compared.

A case is a dict of plain values.  `kind` names the operator:

    prompt   Context.prompt_attend      causal attention over whole prompts in 16 bits that lie packed, one after the other
    append   Context.kv_append_packed   keys and values of packed tokens into a cache in 8 bits
    take     Context.kv_free and Context.kv_take   pages that an eviction took out come back, blocks to come get pages
    fork     Context.kv_fork            sequences become copies of others: shared pages, an open block of their own
    compact  Context.kv_compact         the pages that are in use come to lie at the front of the pool

B sequences, L tokens in the longest (prompts; caches before the call), H key/value heads of D dimensions, g query heads to each of
them, n new tokens of the longest sequence.  `ragged`: the sequences differ in these.

The cache is what a program holds between calls: pages of 64 tokens of one head (e4m3 codes and a power of two as scale, for keys and
for values; the smallest and largest code of every dimension of the keys), a table of pages per sequence and head, the open
block's tokens in 16 bits.  `refs` holds how many entries of the table name a page; 0: it is free.
"""
import math

import torch

own = False

BLOCK = 64
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # one user's short question: latency
        dict(name="prompt_short", kind="prompt", dtype="bf16", B=1, L=77, H=8, g=4, D=128, ragged=False, fused=False),
        # two prompts of 4096 tokens
        dict(name="prompt_pair", kind="prompt", dtype="bf16", B=2, L=4096, H=8, g=4, D=128, ragged=False, fused=False),
        # what a served batch is given at a time: prompts of 1 to 2500 tokens, views of one projection; no size is a multiple of anything
        dict(name="prompt_packed", kind="prompt", dtype="fp16", B=24, L=2500, H=4, g=5, D=96, ragged=True, fused=True),
        # one long document, narrow heads
        dict(name="prompt_long", kind="prompt", dtype="bf16", B=1, L=8192, H=4, g=8, D=64, ragged=False, fused=True),
        # a step that mixes single tokens with the pieces of a few prompts
        dict(name="append_mixed", kind="append", dtype="bf16", B=64, n=300, L=4000, H=8, D=128, ragged=True, mixed=True),
        # prompts of up to 4096 tokens into empty caches
        dict(name="append_prompts", kind="append", dtype="fp16", B=16, n=4096, L=0, H=8, D=128, ragged=True, mixed=False),
        # a step after an eviction: its pages come back, sequences whose block fills up get one
        dict(name="take_step", kind="take", B=64, n=1, L=4000, H=8, ragged=True, spare=500, freed=16),
        # pages for prompts of up to 8192 tokens from a large pool with gaps
        dict(name="take_prompts", kind="take", B=32, n=8192, L=0, H=8, ragged=True, spare=400_000, freed=64),
        # beams of eight requests: two of four go on, each twice
        dict(name="fork_beams", kind="fork", dtype="bf16", B=32, L=2000, H=8, D=128, ragged=True, every=2, cut=False),
        # 63 requests begin with what one sequence holds already
        dict(name="fork_prefix", kind="fork", dtype="bf16", B=64, L=16_000, H=8, D=128, ragged=False, every=64, cut=True),
        # a small pool, a third of it in use
        dict(name="compact_small", kind="compact", dtype="bf16", B=4, L=3000, H=2, D=64, ragged=True, gaps=2.0),
        # 64 sequences of up to 8192 tokens after many others have left
        dict(name="compact_large", kind="compact", dtype="bf16", B=64, L=8192, H=8, D=128, ragged=True, gaps=1.0),
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
        kind = rng.choice(["prompt", "prompt", "prompt", "prompt", "append", "append", "take", "fork", "compact"])
        B, H, ragged = _log(rng, 1, 64), rng.choice([1, 2, 4, 5, 8, 8]), rng.random() < 0.6
        D, dtype = rng.choice([64, 96, 128, 128]), rng.choice(["bf16", "bf16", "fp16"])
        if kind == "prompt":
            g = rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8, 8, 12, 16])
            c = dict(kind=kind, dtype=dtype, B=B, L=_log(rng, 1, 8192), H=H, g=g, D=D, ragged=ragged, fused=rng.random() < 0.5)
            if B * H * g * c["L"] ** 2 > 2 * 32 * 4096 * 4096:  # the plain form's logits
                continue
        elif kind == "append":
            c = dict(kind=kind, dtype=dtype, B=B, n=_log(rng, 1, 4096), L=_log(rng, 1, 8192), H=H, D=D, ragged=ragged, mixed=rng.random() < 0.5)
        elif kind == "take":
            c = dict(kind=kind, B=B, n=_log(rng, 1, 8192), L=_log(rng, 1, 8192), H=H, ragged=ragged, spare=_log(rng, 100, 400_000), freed=_log(rng, 1, 64))
        elif kind == "fork":
            c = dict(kind=kind, dtype=dtype, B=B, L=_log(rng, 1, 16_000), H=H, D=D, ragged=ragged, every=rng.choice([1, 2, 3, 4, 8, B]), cut=rng.random() < 0.5)
        else:
            c = dict(kind=kind, dtype=dtype, B=B, L=_log(rng, 64, 8192), H=H, D=D, ragged=ragged, gaps=rng.choice([0.1, 0.5, 1.0, 2.0]))
        if _cost(c) <= most[kind]:
            return c


def _lens(case):
    """Tokens of every prompt, or in every sequence's cache before the call."""
    B, L = case["B"], case["L"]
    if case["kind"] == "prompt":
        return [max(1, L - (b * 7919) % L) if case["ragged"] else L for b in range(B)]
    return [max(0, L * (b + 1) // B - (b * 13) % 29) if case["ragged"] else L for b in range(B)]


def _counts(case):
    """New tokens of every sequence: of all about as many, or of seven in eight just one (`mixed`)."""
    B, n = case["B"], case["n"]
    counts = [n - (b * 7919) % max(1, 2 * n // 3) if case["ragged"] and n > 1 else n for b in range(B)]
    return [1 if case.get("mixed") and b % 8 else x for b, x in enumerate(counts)]


def _sources(case):
    """The sequence that every sequence becomes a copy of: in groups of `every`, of which the first half goes on (of a group that is cut,
    or of two: the first one)."""
    every = case["every"]
    half = 1 if case["cut"] else max(1, every // 2)
    return [b - b % every + b % every % half for b in range(case["B"])]


def _keep(case):
    """Tokens that a copy takes over, where it is cut."""
    lens = _lens(case)
    return [lens[s] if s == b else lens[s] * 3 // 4 for b, s in enumerate(_sources(case))]


def _used(case):
    """Pages that a compact case has in use, and how many of them lie behind that number as a rule."""
    used = sum(x // BLOCK for x in _lens(case)) * case["H"]
    free = int(used * case["gaps"]) + 1
    return used, free, used * free // max(1, used + free)


def work(case):
    H, kind = case["H"], case["kind"]
    if kind == "prompt":
        lens, g, D = _lens(case), case["g"], case["D"]
        return {"bytes": sum(lens) * H * ((2 * g + 2) * D * 2 + 4 * g), "flops": sum(x * (x + 1) // 2 for x in lens) * H * g * 4 * D}
    lens = _lens(case)
    if kind == "append":
        D, moved, counts = case["D"], 0, _counts(case)
        for x, c in zip(lens, counts):
            full = (x % BLOCK + c) // BLOCK
            left = (x % BLOCK + c) % BLOCK if full else c
            old = x % BLOCK if full else 0  # what the open block held when it fills up
            moved += c * 4 * D + old * 4 * D + full * (BLOCK * 2 * D + 8 + 2 * D) + left * 4 * D
        return {"bytes": H * moved, "flops": H * sum(counts) * 2 * D * 3}
    entries = case["B"] * H * _columns(case)
    if kind == "take":
        return {"bytes": 8 * _pages_of_take(case) + 8 * entries + 4 * case["B"] * H * case["freed"], "flops": 0}
    D = case["D"]
    if kind == "fork":
        moved = 0
        for b, s in enumerate(_sources(case)):
            if s != b:
                keep = _keep(case)[b] if case["cut"] else lens[s]
                moved += keep // BLOCK * 16 + (0 if keep < lens[s] else lens[s] % BLOCK * 8 * D)
        return {"bytes": H * moved + 24 * case["B"], "flops": 0}
    used, free, moving = _used(case)
    return {"bytes": moving * 2 * (BLOCK * 2 * D + 8 + 2 * D) + 8 * (used + free) + 8 * entries, "flops": 0}


def _columns(case):
    most = max(x + y for x, y in zip(_lens(case), _counts(case))) if "n" in case else max(_lens(case))
    return most // BLOCK + 1


def _pages_of_take(case):
    full = sum(x // BLOCK for x in _lens(case))
    to_come = sum((x + y) // BLOCK - x // BLOCK for x, y in zip(_lens(case), _counts(case)))
    return (full + to_come + case["B"] * case["freed"]) * case["H"] + case["spare"]


# ---- inputs


def _seal(x):
    """Blocks [..., 64, D] in float32 as codes and scales: the smallest power of two that leaves every value within 448."""
    m, e = torch.frexp(x.abs().amax((-1, -2)))
    e = (e - torch.where(m <= 0.875, 9, 8)).clamp(-126, 119)
    scale = torch.ldexp(torch.ones_like(m), torch.where(m > 0, e, 0))
    return (x / scale[..., None, None]).to(torch.float8_e4m3fn), scale


def _table(case, lens, columns, pages, rand):
    """A table whose blocks have pages in random order, and how often each page stands in it."""
    B, H, dev = case["B"], case["H"], "cuda"
    order = torch.randperm(pages, generator=rand, device=dev).to(torch.int32)
    full = torch.tensor(lens, device=dev)[:, None, None] // BLOCK
    has = (torch.arange(columns, device=dev) < full).expand(B, H, columns)
    table = torch.full((B, H, columns), -1, device=dev, dtype=torch.int32)
    table[has] = order[: int(has.sum())]
    refs = torch.zeros(pages, device=dev, dtype=torch.int32)
    refs[table[has].long()] = 1
    return table, refs, order[int(has.sum()) :]


def _cache(case, lens, room, pages, rand):
    """A cache with `lens` tokens whose table has room for `room` more in every sequence."""
    B, H, D, T = case["B"], case["H"], case["D"], TYPES[case["dtype"]]
    dev = "cuda"
    columns = max((x + r) // BLOCK for x, r in zip(lens, room)) + 1
    table, refs, _ = _table(case, lens, columns, pages, rand)
    codes = lambda *shape: torch.randn(shape, generator=rand, device=dev, dtype=torch.bfloat16).mul_(64).to(torch.float8_e4m3fn)  # noqa: E731
    c = dict(k=codes(pages, BLOCK, D), v=codes(pages, D, BLOCK), scales=torch.exp2(torch.randint(-8, -4, (pages, 2), generator=rand, device=dev).float()),
             bounds=codes(pages, 2, D), tail_k=torch.randn(B, H, 2, BLOCK, D, generator=rand, device=dev).to(T),
             tail_v=torch.randn(B, H, 2, D, BLOCK, generator=rand, device=dev).to(T), table=table,
             lens=torch.tensor(lens, device=dev, dtype=torch.int32), evicted=torch.randint(0, 2, (B,), generator=rand, device=dev, dtype=torch.int32))
    return c, refs


def _starts(lens):
    return torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)


def prepare(case, seed):
    rand = torch.Generator(device="cuda")
    rand.manual_seed(int(seed))
    dev, B, H, kind, lens = "cuda", case["B"], case["H"], case["kind"], _lens(case)
    s = dict(case=case)
    if kind == "prompt":
        g, D, T = case["g"], case["D"], TYPES[case["dtype"]]
        n = sum(lens)
        # keys follow topics, and queries ask for one
        topics = torch.randn(32, H, 1, D, generator=rand, device=dev)
        qkv = torch.randn(n, H * (g + 2), D, generator=rand, device=dev)
        qkv[:, : H * g].view(n, H, g, D).add_(topics[torch.randint(0, 32, (n,), generator=rand, device=dev)])
        qkv[:, H * g : H * (g + 1)].view(n, H, 1, D).add_(topics[torch.randint(0, 32, (n // BLOCK + 1,), generator=rand, device=dev).repeat_interleave(BLOCK)[:n]], alpha=0.8)
        qkv = qkv.to(T)
        s["q"], s["k"], s["v"] = (x if case["fused"] else x.contiguous() for x in qkv.split([H * g, H, H], 1))
        s["starts"], s["longest"] = _starts(lens), max(lens)
        return s
    if kind == "append":
        counts, D, T = _counts(case), case["D"], TYPES[case["dtype"]]
        pages = H * sum((x + r) // BLOCK for x, r in zip(lens, counts)) + 3
        s["cache"], _ = _cache(case, [x + y for x, y in zip(lens, counts)], [0] * B, pages, rand)
        s["cache"]["lens"].copy_(torch.tensor(lens))
        spread = torch.exp(0.5 * torch.randn(2, 1, H, D, generator=rand, device=dev))
        s["k"], s["v"] = ((spread[i] * torch.randn(sum(counts), H, D, generator=rand, device=dev)).to(T) for i in range(2))
        s["starts"], s["longest"] = _starts(counts), max(counts)
        return s
    if kind == "take":
        counts = _counts(case)
        pages = _pages_of_take(case)
        table, s["refs"], others = _table(case, lens, _columns(case), pages, rand)
        # an eviction's pages, as it leaves them: a row's first ones, then -1; and pages that others hold
        s["freed"] = torch.full((B, H, table.shape[2] + case["freed"]), -1, device=dev, dtype=torch.int32)
        s["freed"][:, :, : case["freed"]] = others[: B * H * case["freed"]].view(B, H, case["freed"])
        s["refs"][s["freed"][:, :, : case["freed"]].long()] = 1
        held = others[B * H * case["freed"] :]
        s["refs"][held[: case["spare"] // 2].long()] = 1
        s["table"], s["lens"], s["counts"] = table, torch.tensor(lens, device=dev, dtype=torch.int32), torch.tensor(counts, device=dev, dtype=torch.int32)
        # a cache of the smallest pages: the call reads the table and the lengths only
        s["rest"] = dict(k=torch.zeros(pages, BLOCK, 64, device=dev, dtype=torch.float8_e4m3fn), v=torch.zeros(pages, 64, BLOCK, device=dev, dtype=torch.float8_e4m3fn),
                         scales=torch.ones(pages, 2, device=dev), bounds=torch.zeros(pages, 2, 64, device=dev, dtype=torch.float8_e4m3fn),
                         tail_k=torch.zeros(B, H, 2, BLOCK, 64, device=dev, dtype=torch.bfloat16), tail_v=torch.zeros(B, H, 2, 64, BLOCK, device=dev, dtype=torch.bfloat16),
                         evicted=torch.zeros(B, device=dev, dtype=torch.int32))
        return s
    if kind == "fork":
        s["cache"], s["refs"] = _cache(case, lens, [0] * B, H * sum(x // BLOCK for x in lens) + 5, rand)
        s["source"] = torch.tensor(_sources(case), device=dev, dtype=torch.int32)
        s["keep"] = torch.tensor(_keep(case), device=dev, dtype=torch.int32) if case["cut"] else None
        return s
    used, free, _ = _used(case)
    s["cache"], s["refs"] = _cache(case, lens, [0] * B, used + free, rand)
    # one block in eight is shared by the sequence after it
    table, shared = s["cache"]["table"], torch.rand(s["cache"]["table"].shape, generator=rand, device=dev) < 0.125
    shared[0] = False
    before = table.roll(1, 0)
    shared &= (table >= 0) & (before >= 0)
    s["cache"]["table"] = torch.where(shared, before, table)
    s["refs"] = torch.bincount(s["cache"]["table"].flatten().long() + 1, minlength=used + free + 1)[1:].to(torch.int32)
    return s


# ---- the operators


def run(state):
    return _own_run(state) if own else _plain_run(state)


def _own_run(s):
    import paper_1509_05186_amd as etf

    kind = s["case"]["kind"]
    if "context" not in s:
        s["context"] = etf.Context(device=0, stream=torch.cuda.current_stream().cuda_stream)
        if kind == "take":
            s["handle"] = etf.KvCache(table=s["table"], lens=s["lens"], **s["rest"])
        elif kind != "prompt":
            s["handle"] = etf.KvCache(**s["cache"])
    ctx = s["context"]
    if kind == "prompt":
        lse = torch.empty(s["q"].shape[:2], device=s["q"].device)
        return {"out": ctx.prompt_attend(s["q"], s["k"], s["v"], s["starts"], lse=lse), "lse": lse}
    if kind == "append":
        ctx.kv_append_packed(s["handle"], s["k"], s["v"], s["starts"])
        return {x: s["cache"][x] for x in ("k", "v", "scales", "bounds", "tail_k", "tail_v")}
    if kind == "take":
        ctx.kv_free(s["refs"], s["freed"])
        table, refs = torch.empty_like(s["table"]), torch.empty_like(s["refs"])
        missing = ctx.kv_take(s["handle"], s["refs"], s["case"]["n"], counts=s["counts"], table_out=table, refs_out=refs)
        return {"table": table, "refs": refs, "missing": missing}
    if kind == "fork":
        ctx.kv_fork(s["handle"], s["refs"], s["source"], keep=s["keep"])
        return dict({x: s["cache"][x] for x in ("table", "lens", "evicted", "tail_k", "tail_v")}, refs=s["refs"])
    table, refs = torch.empty_like(s["cache"]["table"]), torch.empty_like(s["refs"])
    used = ctx.kv_compact(s["handle"], s["refs"], table_out=table, refs_out=refs)
    return dict({x: s["cache"][x] for x in ("k", "v", "scales", "bounds")}, table=table, refs=refs, used=used)


def _plain_run(s):
    kind = s["case"]["kind"]
    if kind == "prompt":
        return _plain_prompt(s["q"], s["k"], s["v"], s["starts"], s["longest"])
    if kind == "append":
        return _plain_append(s["cache"], s["k"], s["v"], s["starts"], s["longest"])
    if kind == "take":
        _plain_free(s["refs"], s["freed"])
        return _plain_take(s["table"], s["lens"], s["refs"], s["counts"])
    if kind == "fork":
        return _plain_fork(s["cache"], s["refs"], s["source"], s["keep"])
    return _plain_compact(s["cache"], s["refs"])


def _padded(x, starts, longest):
    """Packed rows as [B, longest, ...] (what lies behind a sequence's end: its last row, or any), and each place's row."""
    at = starts[:-1, None].long() + torch.arange(longest, device=x.device)
    at = torch.minimum(at, (starts[1:, None].long() - 1)).clamp_min(0)
    return x[at], at


def _plain_prompt(q, k, v, starts, longest):
    n, Hq, D = q.shape
    H, g = k.shape[1], Hq // k.shape[1]
    Q, at = _padded(q, starts, longest)
    K, V = _padded(k, starts, longest)[0], _padded(v, starts, longest)[0]
    B, i = len(Q), torch.arange(longest, device=q.device)
    rows = Q.view(B, longest, H, g, D).permute(0, 2, 3, 1, 4).reshape(B, H, g * longest, D).float()
    logits = (rows @ K.permute(0, 2, 3, 1).float()).mul_(1 / math.sqrt(D)).view(B, H, g, longest, longest)
    logits.masked_fill_(i > i[:, None], -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = logits.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p.view(B, H, g * longest, longest) @ V.transpose(1, 2).float()).view(B, H, g, longest, D) / total
    lse = (top + total.log())[..., 0]
    # every row from its place: the last place of a sequence's padding is the same row as its end, so only true places are taken
    seq = torch.searchsorted(starts[1:].contiguous(), torch.arange(n, device=q.device, dtype=torch.int32), right=True)
    place = torch.arange(n, device=q.device) - starts.long()[seq]
    out = out.permute(0, 3, 1, 2, 4)[seq, place].reshape(n, Hq, D).to(q.dtype)
    return {"out": out, "lse": lse.permute(0, 3, 1, 2)[seq, place].reshape(n, Hq)}


def _plain_append(c, k, v, starts, n):
    counts = (starts[1:] - starts[:-1]).long()
    k, v = _padded(k, starts, n)[0], _padded(v, starts, n)[0]
    B, _, H, D = k.shape
    dev = k.device
    lens = c["lens"].long()
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


def _plain_free(refs, pages):
    """One share less of each listed page, none below zero."""
    gone = torch.zeros(len(refs) + 1, device=refs.device, dtype=torch.int32)
    at = torch.where((pages >= 0) & (pages < len(refs)), pages, len(refs)).flatten().long()
    gone.scatter_add_(0, at, torch.ones_like(at, dtype=torch.int32))
    refs.copy_((refs - gone[:-1]).clamp_min(0))


def _plain_take(table, lens, refs, counts):
    pages, dev = len(refs), table.device
    j = torch.arange(table.shape[2], device=dev)
    lens, counts = lens.long()[:, None, None], counts.long()[:, None, None]
    there = (table >= 0) & (table < pages)
    shares = torch.where(there, refs[table.clamp(0, pages - 1).long()], 0)
    need = (j >= lens // BLOCK) & (j < (lens + counts) // BLOCK) & (shares != 1)
    free = refs <= 0
    missing = (need.sum() - free.sum()).clamp_min(0)
    # free pages by number, and which of them every block takes
    rank = torch.where(free, free.cumsum(0) - 1, pages)
    lowest = torch.empty(pages + 1, device=dev, dtype=torch.int32).scatter_(0, rank, torch.arange(pages, device=dev, dtype=torch.int32))
    mine = need.flatten().cumsum(0).view(need.shape) - 1
    got = need & (missing == 0)
    new = torch.where(got, lowest[mine.clamp(0, pages - 1)], table)
    change = torch.zeros(pages + 1, device=dev, dtype=torch.int32)
    change.scatter_add_(0, torch.where(got & (shares > 1), table, pages).flatten().long(), torch.full_like(table, -1).flatten())
    change.scatter_add_(0, torch.where(got, new, pages).flatten().long(), torch.ones_like(table).flatten())
    return {"table": new, "refs": refs + change[:-1], "missing": missing.to(torch.int32).view(1)}


def _plain_fork(c, refs, source, keep):
    table, lens, evicted = c["table"], c["lens"], c["evicted"]
    B, H, blocks = table.shape
    pages, dev = len(refs), table.device
    batch, j, t = torch.arange(B, device=dev), torch.arange(blocks, device=dev), torch.arange(BLOCK, device=dev)
    src = source.long()
    from_lens = lens[src].long()
    whole = from_lens if keep is None else torch.where(keep >= from_lens, from_lens, keep.long().clamp_min(0) // BLOCK * BLOCK)
    stays = ((src == batch) & (whole == from_lens))[:, None, None]
    new = torch.where(stays, table, torch.where(j < (whole // BLOCK)[:, None, None], table[src], -1))
    change = torch.zeros(pages + 1, device=dev, dtype=torch.int32)
    for x, sign in ((table, -1), (new, 1)):
        at = torch.where((x >= 0) & (x < pages) & ~stays, x, pages).flatten().long()
        change.scatter_add_(0, at, torch.full_like(at, sign, dtype=torch.int32))
    refs.add_(change[:-1])
    # the open block's tokens, in the same of the two buffers
    buf = (from_lens // BLOCK + evicted[src].long()) % 2
    copied = t < torch.where(whole == from_lens, from_lens % BLOCK, 0)[:, None]
    for tail, mask in ((c["tail_k"], copied[:, None, :, None]), (c["tail_v"], copied[:, None, None, :])):
        tail[batch, :, buf] = torch.where(mask, tail[src, :, buf], tail[batch, :, buf])
    table.copy_(new)
    evicted.copy_(evicted[src])
    lens.copy_(whole)
    return dict({x: c[x] for x in ("table", "lens", "evicted", "tail_k", "tail_v")}, refs=refs)


def _plain_compact(c, refs):
    pages, dev = len(refs), refs.device
    used = refs > 0
    many, upto, page = used.sum(), used.cumsum(0), torch.arange(pages, device=dev)
    hole, moves = ~used & (page < many), used & (page >= many)
    # the i-th hole takes the used page that has i used ones behind it
    of_rank = torch.empty(pages + 1, device=dev, dtype=torch.long).scatter_(0, torch.where(hole, page - upto, pages), page)
    to = torch.where(moves, of_rank[many - upto], page)
    old = page[moves]
    new = to[old]
    for x in ("k", "v", "scales", "bounds"):
        c[x][new] = c[x][old]
    after = torch.zeros_like(refs).scatter_(0, to, torch.where(used, refs, 0), reduce="add")
    there = (c["table"] >= 0) & (c["table"] < pages)
    table = torch.where(there, to[c["table"].clamp(0, pages - 1).long()].to(torch.int32), c["table"])
    return dict({x: c[x] for x in ("k", "v", "scales", "bounds")}, table=table, refs=after, used=many.to(torch.int32).view(1))


# ---- the definitions in 64 bits


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "prompt":
        return _exact_prompt(case, s)
    if kind == "append":
        return _exact_append(case, s)
    if kind == "fork":
        return _exact_fork(case, s)
    if kind == "compact":
        return _exact_compact(s)
    return None  # whole numbers


def _exact_prompt(case, s):
    H, g, D = case["H"], case["g"], case["D"]
    if work(case)["flops"] > 3e12:
        return None
    q, k, v, at = s["q"], s["k"], s["v"], s["starts"].tolist()
    out = torch.zeros(q.shape, device=q.device, dtype=torch.float64)
    lse = torch.zeros(q.shape[:2], device=q.device, dtype=torch.float64)
    for a, z in zip(at, at[1:]):
        step = max(1, min(z - a, 100_000_000 // (z - a)))
        for x in range(H * g):
            kk, vv = k[a:z, x // g].double(), v[a:z, x // g].double()
            for i in range(a, z, step):
                rows = q[i : min(z, i + step), x].double() @ kk.T / math.sqrt(D)
                sees = torch.arange(a, z, device=q.device) <= torch.arange(i, i + len(rows), device=q.device)[:, None]
                rows = torch.where(sees, rows, -math.inf)
                lse[i : i + len(rows), x] = torch.logsumexp(rows, 1)
                out[i : i + len(rows), x] = torch.softmax(rows, 1) @ vv
    return {"out": out, "lse": lse}


def _exact_round(x):
    """Blocks x [N, 64, D] in float64 as e4m3 values (float64) and their scales: three bits after the leading one, steps of 2^-9 at least."""
    most = x.abs().amax((1, 2))
    e = torch.where(most > 0, torch.ceil(torch.log2(most.clamp_min(2.0**-200) / 448)), 0)
    e = torch.where(448 * torch.exp2(e) < most, e + 1, torch.where((448 * torch.exp2(e - 1) >= most) & (most > 0), e - 1, e)).clamp(-126, 119)
    y = x / torch.exp2(e)[:, None, None]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0**-6))) - 3)
    return torch.round(y / step) * step, torch.exp2(e)


def _exact_append(case, s):
    if case["B"] * case["H"] > 600 or len(s["k"]) * case["H"] > 400_000:
        return None
    c, at = s["cache"], s["starts"].tolist()
    lens, evicted = c["lens"].tolist(), c["evicted"].tolist()
    got = {x: c[x].double() for x in ("k", "v", "scales", "bounds", "tail_k", "tail_v")}
    for b in range(case["B"]):
        first, begin = divmod(lens[b], BLOCK)
        for h in range(case["H"]):
            buf = (first + evicted[b]) % 2
            k = torch.cat([c["tail_k"][b, h, buf, :begin], s["k"][at[b] : at[b + 1], h]]).double()
            v = torch.cat([c["tail_v"][b, h, buf, :, :begin].T, s["v"][at[b] : at[b + 1], h]]).double()
            whole, left = divmod(len(k), BLOCK)
            if whole:
                page = c["table"][b, h, first : first + whole].long()
                codes, got["scales"][page, 0] = _exact_round(k[: whole * BLOCK].view(whole, BLOCK, -1))
                got["k"][page], got["bounds"][page, 0], got["bounds"][page, 1] = codes, codes.amin(1), codes.amax(1)
                codes, got["scales"][page, 1] = _exact_round(v[: whole * BLOCK].view(whole, BLOCK, -1))
                got["v"][page] = codes.transpose(1, 2)
            buf = (first + whole + evicted[b]) % 2
            got["tail_k"][b, h, buf, :left] = k[whole * BLOCK :]
            got["tail_v"][b, h, buf, :, :left] = v[whole * BLOCK :].T
    return got


def _exact_fork(case, s):
    c = s["cache"]
    lens, evicted, source = c["lens"].tolist(), c["evicted"].tolist(), s["source"].tolist()
    keep = lens if s["keep"] is None else s["keep"].tolist()
    got = {x: c[x].double() for x in ("tail_k", "tail_v")}
    for b, x in enumerate(source):
        left = lens[x] % BLOCK
        if x != b and left and (s["keep"] is None or keep[b] >= lens[x]):
            buf = (lens[x] // BLOCK + evicted[x]) % 2
            got["tail_k"][b, :, buf, :left] = c["tail_k"][x, :, buf, :left].double()
            got["tail_v"][b, :, buf, :, :left] = c["tail_v"][x, :, buf, :, :left].double()
    return dict(table=None, lens=None, evicted=None, refs=None, **got)


def _exact_compact(s):
    c = s["cache"]
    if c["k"].numel() > 300_000_000:
        return None
    shares = s["refs"].tolist()
    used = [p for p, n in enumerate(shares) if n > 0]
    holes = [p for p, n in enumerate(shares[: len(used)]) if n <= 0]
    movers = [p for p in reversed(used) if p >= len(used)]
    old, new = (torch.tensor(x, device=c["k"].device, dtype=torch.long) for x in (movers, holes))
    got = {x: c[x].double() for x in ("k", "v", "scales", "bounds")}
    for x in got.values():
        x[new] = x[old]
    return dict(table=None, refs=None, used=None, **got)
