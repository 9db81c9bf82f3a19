"""Evictions from a table whose pages are counted, on the GPU: pages that were taken ahead of their tokens, or that a draft has left behind, stay in
the table or are named as freed, so that shares and entries agree.  Whole numbers and copies, equal to the last bit."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import kvcache as kv, pages as pg  # noqa: E402
import paper_1509_05186_amd as etf  # noqa: E402

BF, HF = torch.bfloat16, torch.float16


def say(*a):
    print(*a, flush=True)


def context():
    return etf.Context(device=0, stream=torch.cuda.current_stream().cuda_stream)


def on_gpu(c):
    return etf.KvCache(**{name: c[name].cuda() for name in etf.KvCache.FIELDS})


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def shares_agree(cache, refs):
    c = {name: getattr(cache, name).cpu() for name in etf.KvCache.FIELDS}
    return torch.equal(pg.count(c), refs.cpu())


# tables on both sides of every kernel's limit, full to the end, of empty sequences, with budgets that take something out and that do not
@pytest.mark.parametrize("blocks,lens,budget,sink,recent", [(8, [500, 64, 0, 130], 4, 1, 1), (1, [64], 1, 0, 0), (1, [0], 3, 1, 1), (12, [64 * 12 + 63, 64 * 11], 5, 0, 0), (8, [300], 8, 1, 1),
                                                            (256, [64 * 200 + 5, 64], 100, 2, 3), (257, [64 * 130, 64 * 257], 100, 2, 3), (1024, [64 * 700], 650, 4, 8), (1025, [64 * 700 + 1], 64, 4, 8),
                                                            (4097, [64 * 3000 + 9], 1000, 0, 5), (17_000, [64 * 9000 + 9], 700, 3, 20)])
def test_evict_ahead(blocks, lens, budget, sink, recent):
    say("evict ahead", blocks, lens, budget, sink, recent)
    B, H = len(lens), 2
    g = torch.Generator().manual_seed(blocks + budget)
    c = kv.new_cache(B, H, 64, blocks, BF, pages=5, table=torch.randint(-2, 1 << 20, (B, H, blocks), generator=g))
    c["lens"].copy_(torch.tensor(lens))
    c["evicted"].copy_(torch.randint(0, 9, (B,), generator=g))
    mass = torch.randint(0, 50, (B, H, blocks), generator=g).float()
    if blocks > 8:
        mass[0, 1, 3], mass[0, 1, 4] = math.nan, math.inf
    want = pg.evict(c, mass, budget, sink, recent)
    same = lambda got: all(torch.equal(torch.nan_to_num(x.cpu(), nan=-9.0), torch.nan_to_num(y, nan=-9.0)) for x, y in zip(got, want))  # noqa: E731
    ctx, cache = context(), on_gpu(c)
    to = cache.fork()
    kept, freed = ctx.kv_evict(cache, mass.cuda(), budget, sink=sink, recent=recent, to=to, ahead=True)
    assert same((to.table, to.lens, to.evicted, kept, freed))
    assert torch.equal(cache.table.cpu(), c["table"])
    if blocks <= 16384:
        own = mass.cuda()
        _, freed = ctx.kv_evict(cache, own, budget, sink=sink, recent=recent, ahead=True)
        assert same((cache.table, cache.lens, cache.evicted, own, freed))


@pytest.mark.parametrize("dtype,D", [(BF, 64), (HF, 128)])
@pytest.mark.parametrize("budget", [20, 5, 3])
def test_pages_taken_ahead_outlive_an_eviction(dtype, D, budget):
    """Pages for the next 64 tokens, some of these tokens, an eviction, the others: no page is lost, and the tokens find theirs."""
    say("taken ahead", dtype, D, budget)
    B, H, g, blocks = 3, 2, 2, 12
    gen = torch.Generator().manual_seed(D + budget)
    rand = lambda *s: torch.randn(s, generator=gen).to(dtype).cuda()  # noqa: E731
    ctx = context()
    pool = etf.KvCache.alloc(B, H, D, blocks * 64, dtype=dtype, pages=200)
    plain = etf.KvCache.alloc(B, H, D, blocks * 64, dtype=dtype)
    refs = torch.zeros(200, dtype=torch.int32, device="cuda")
    counts, held = [330, 64, 47], plain.pages

    def come(n, counts=None):
        k, v = rand(B, n, H, D), rand(B, n, H, D)
        for cache in (pool, plain):
            ctx.kv_append(cache, k, v, counts=counts)
            cache.lens += n if counts is None else counts

    assert int(ctx.kv_take(pool, refs, 330, counts=ints(counts))) == 0
    come(330, ints(counts))
    for turn in range(3):
        assert int(ctx.kv_take(pool, refs, 64)) == 0
        in_use = int((refs > 0).sum())
        come(13)
        mass = torch.rand(B, H, blocks, generator=gen).cuda()
        _, freed = ctx.kv_evict(pool, mass.clone(), budget, sink=1, recent=1, ahead=True)
        ctx.kv_free(refs, freed)
        ctx.kv_evict(plain, mass.clone(), budget, sink=1, recent=1, ahead=True)
        assert shares_agree(pool, refs) and int((refs > 0).sum()) == in_use - int((freed >= 0).sum())
        # its rows of the table have lost pages; what it has left serves the tokens of this test
        assert int((plain.table >= 0).sum()) == held - int((freed >= 0).sum())
        held = int((plain.table >= 0).sum())
        come(51)     # the rest of the 64, into the pages that were taken before the eviction
        q = rand(B, 1, H * g, D)
        assert torch.equal(ctx.kv_attend(pool, q), ctx.kv_attend(plain, q)), turn
        assert shares_agree(pool, refs)
    # everybody leaves: every page is free
    ctx.kv_fork(pool, refs, ints([-1] * B))
    assert not refs.any()


def test_a_page_of_a_draft_that_was_taken_back():
    say("draft, eviction")
    D, H = 96, 2
    gen = torch.Generator().manual_seed(3)
    rand = lambda n: torch.randn(1, n, H, D, generator=gen).to(HF).cuda()  # noqa: E731
    ctx = context()
    pool = etf.KvCache.alloc(1, H, D, 640, dtype=HF, pages=30)
    refs = torch.zeros(30, dtype=torch.int32, device="cuda")

    def come(n):
        k, v = rand(n), rand(n)
        assert int(ctx.kv_take(pool, refs, n)) == 0
        ctx.kv_append(pool, k, v)
        pool.lens += n

    come(64 * 4 + 60)
    come(10)
    pool.lens -= 10     # the block that the draft completed is open again, and its page is in the table
    q = torch.randn(1, 1, 2 * H, D, generator=gen).to(HF).cuda()
    mass = torch.rand(1, H, pool.max_blocks, generator=gen).cuda()
    for budget in (6, 2):
        _, freed = ctx.kv_evict(pool, mass.clone(), budget, ahead=True)
        ctx.kv_free(refs, freed)
        assert shares_agree(pool, refs) and int((pool.table >= 0).sum()) == H * (min(4, budget) + 1)
    assert pool.lens.tolist() == [2 * 64 + 60] and pool.evicted.tolist() == [2]
    page = pool.table[:, :, 2].clone()
    come(5)
    assert torch.equal(pool.table[:, :, 2], page) and shares_agree(pool, refs) and pool.lens.tolist() == [3 * 64 + 1]
    assert torch.isfinite(ctx.kv_attend(pool, q)).all()


def test_in_a_graph():
    """Captured and replayed, with the same call between the replays."""
    say("evict ahead: graph")
    g = torch.Generator().manual_seed(9)
    c = kv.new_cache(2, 3, 64, 300, BF, pages=5, table=torch.randint(-1, 5000, (2, 3, 300), generator=g))
    c["lens"].copy_(torch.tensor([64 * 200 + 3, 64 * 20]))
    mass = torch.rand(2, 3, 300, generator=g)
    want = pg.evict(c, mass, 50, 1, 2)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        cache, own, freed = on_gpu(c), mass.cuda(), torch.empty(2, 3, 300, dtype=torch.int32, device="cuda")
        ctx = etf.Context(device=0, stream=side.cuda_stream)

        def step():
            ctx.kv_evict(cache, own, 50, sink=1, recent=2, freed=freed, ahead=True)

        def restore():
            for name in ("table", "lens", "evicted"):
                getattr(cache, name).copy_(c[name])
            own.copy_(mass)
            freed.fill_(7)

        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        for i in range(3):
            for way in (graph.replay, step):
                restore()
                way()
                side.synchronize()
                for x, y in zip((cache.table, cache.lens, cache.evicted, own, freed), want):
                    assert torch.equal(x.cpu(), y), i
