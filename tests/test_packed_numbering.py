"""The numbering of packed sequences' tiles, worked out as the kernels do it: where starts ascend, every tile has one number of those that a launch has;
whatever starts are, a number stands for a tile that its sequence has, or for none, and no tile has two.  On the GPU: calls with starts that descend."""
import random

import pytest

torch = pytest.importorskip("torch")


def tiles_of(starts, tokens, rows, g):
    """{number: (sequence, tile)} over all numbers of a launch."""
    batch = len(starts) - 1
    at = [min(max(s, 0), tokens) for s in starts]
    base = lambda b: at[b] * g // rows + b  # noqa: E731
    got = {}
    for number in range(tokens * g // rows + batch):
        lo, many = 0, batch
        while many > 1:     # 64 places at a time
            step = (many + 63) // 64
            before = [i for i in range(0, many, step) if base(min(lo + i, batch - 1)) <= number]
            last = before[-1] // step if before else 0
            lo, many = lo + last * step, min(step, many - last * step)
        n, tile = at[lo + 1] - at[lo], number - base(lo)
        if n > 0 and tile >= 0 and tile * rows < n * g:
            got[number] = (lo, tile)
    return got, at


@pytest.mark.parametrize("rows,g", [(64, 1), (128, 1), (128, 5), (128, 129), (128, 16)])
def test_ascending_starts(rows, g):
    rng = random.Random(rows + g)
    for batch in (1, 2, 5, 63, 64, 65, 130, 4200):
        for spread in (3, 200, 2000):
            if batch * spread * g > 2_000_000:
                continue
            lens = [rng.choice([0, 0, 1, 63, 64, 65, rng.randrange(spread + 1)]) for _ in range(batch)]
            first, behind = rng.randrange(100), rng.randrange(100)
            starts = [first]
            for n in lens:
                starts.append(starts[-1] + n)
            got, _ = tiles_of(starts, starts[-1] + behind + 1, rows, g)
            want = [(b, t) for b, n in enumerate(lens) for t in range(-(-n * g // rows))]
            assert sorted(got.values()) == want


@pytest.mark.parametrize("rows,g", [(64, 1), (128, 5)])
def test_any_starts(rows, g):
    rng = random.Random(rows)
    for batch in (1, 2, 5, 64, 65, 200):
        for _ in range(20):
            tokens = rng.randrange(1, 3000)
            starts = [rng.randrange(-50, tokens + 50) for _ in range(batch + 1)]
            got, at = tiles_of(starts, tokens, rows, g)
            assert len(set(got.values())) == len(got)
            for b, t in got.values():
                assert 0 <= t * rows < (at[b + 1] - at[b]) * g


def say(*a):
    print(*a, flush=True)


@pytest.mark.gpu
def test_prompts_with_starts_that_descend():
    import paper_1509_05186_amd as etf
    say("prompts, starts that descend")
    T, lead, D, H, g = 1100, 64, 64, 2, 3
    gen = torch.Generator(device="cuda").manual_seed(1)
    made = lambda heads: torch.randn(T + 2 * lead, heads, D, generator=gen, device="cuda").bfloat16()  # noqa: E731
    q, k, v = made(H * g), made(H), made(H)
    for x in (k, v):     # none of these is read
        x[:lead], x[lead + T :] = float("nan"), float("nan")
    ctx = etf.Context(device=0, stream=torch.cuda.current_stream().cuda_stream)
    for starts in ([0, 1000, 50, 1100], [500, 0, 300, 100, 1100], [1100, 0], [640, 300, 700, -5, 1 << 30]):
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
        mid = slice(lead, lead + T)
        ctx.prompt_attend(q[mid], k[mid], v[mid], torch.tensor(starts, dtype=torch.int32, device="cuda"), out=out[mid], lse=lse[mid])
        torch.cuda.synchronize()
        for x in (out, lse):
            assert (x[:lead] == 7).all() and (x[lead + T :] == 7).all() and torch.isfinite(x).all(), starts


@pytest.mark.gpu
def test_appends_with_starts_that_descend():
    import paper_1509_05186_amd as etf
    say("appends, starts that descend")
    T, H, D, pages = 1100, 2, 64, 400
    gen = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn(T, H, D, generator=gen, device="cuda").bfloat16() for _ in range(2))
    ctx = etf.Context(device=0, stream=torch.cuda.current_stream().cuda_stream)
    for starts in ([0, 1000, 50, 1100], [500, 0, 300, 100], [640, 300, 700, -5]):
        cache = etf.KvCache.alloc(3, H, D, 64 * 20, pages=pages)
        cache.table.copy_((torch.randperm(pages, generator=torch.Generator().manual_seed(3)).int()[: 3 * H * 20]).view(3, H, 20))
        cache.k.view(torch.uint8).fill_(0x11)
        ctx.kv_append_packed(cache, k, v, torch.tensor(starts, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        at = [min(max(x, 0), T) for x in starts]
        may = {int(p) for b in range(3) for h in range(H) for p in cache.table[b, h, : max(0, at[b + 1] - at[b]) // 64].tolist()}
        changed = set((cache.k.view(torch.uint8) != 0x11).flatten(1).any(1).nonzero().flatten().tolist())
        assert changed <= may, starts
        for b in range(3):
            if at[b + 1] <= at[b]:
                assert not cache.tail_k[b].any(), starts
