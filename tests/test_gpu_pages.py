"""Pages of the attention cache on the GPU against the oracle (oracle/pages.py): whole numbers and copies, equal to the last bit."""
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


def bits(t):
    return t.cpu().contiguous().view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t.cpu().contiguous().view(torch.int16) if t.element_size() == 2 else t.cpu().contiguous().view(torch.int32)


def same(got, want, what, fields=etf.KvCache.FIELDS):
    for name in fields:
        assert torch.equal(bits(getattr(got, name)), bits(want[name])), "%s: %s" % (what, name)


def a_cache(lens, H, D, blocks, spare, seed=0, dtype=BF, shared=0.0):
    """An oracle's cache whose full blocks have pages in random order among `spare` free ones, contents random bits; (cache, refs)."""
    g = torch.Generator().manual_seed(seed)
    B = len(lens)
    full = [min(n, blocks * 64 + 63) // 64 for n in lens]
    pages = H * sum(full) + spare
    order = torch.randperm(pages, generator=g)
    table, at = torch.full((B, H, blocks), -1, dtype=torch.int32), 0
    for b in range(B):
        table[b, :, : full[b]] = order[at : at + H * full[b]].view(H, full[b])
        at += H * full[b]
    for b in range(1, B):     # some blocks are the sequence's before it
        n = min(full[b], full[b - 1])
        take = torch.rand(H, n, generator=g) < shared
        table[b, :, :n] = torch.where(take, table[b - 1, :, :n], table[b, :, :n])
    c = kv.new_cache(B, H, D, blocks, dtype, pages=max(1, pages), table=table)
    for name in ("k", "v", "bounds"):
        c[name] = torch.randint(0, 256, c[name].shape, generator=g, dtype=torch.uint8).view(torch.float8_e4m3fn)
    c["scales"] = torch.exp2(torch.randint(-9, 9, c["scales"].shape, generator=g).float())
    for name in ("tail_k", "tail_v"):
        c[name] = torch.randint(-(1 << 15), 1 << 15, c[name].shape, generator=g, dtype=torch.int16).view(dtype)
    c["lens"].copy_(torch.tensor(lens))
    c["evicted"].copy_(torch.randint(0, 5, (B,), generator=g))
    return c, pg.count(c)


# ---- take


def check_take(c, refs, n, counts, what):
    say("take", what)
    table, after, missing = pg.take(c, refs, n, counts)
    ctx = context()
    cnt = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    for apart in (True, False):
        cache, r = on_gpu(c), refs.cuda()
        t_out, r_out = (torch.full_like(cache.table, 77), torch.full_like(r, 77)) if apart else (None, None)
        lack = ctx.kv_take(cache, r, n, counts=cnt, table_out=t_out, refs_out=r_out)
        torch.cuda.synchronize()
        assert int(lack) == missing, what
        assert torch.equal((t_out if apart else cache.table).cpu(), table) and torch.equal((r_out if apart else r).cpu(), after), "%s apart %s" % (what, apart)
        if apart:
            same(cache, c, what)
            assert torch.equal(r.cpu(), refs), what
    return table, after, missing


@pytest.mark.parametrize("lens,n,counts", [([0], 1, None), ([63], 1, None), ([0, 63, 64, 127], 1, None), ([10, 70, 200], 64, [64, 0, 53]), ([0, 5, 640], 1000, [1000, 640, 59]),
                                           ([63] * 70, 2, [b % 3 for b in range(70)])])
@pytest.mark.parametrize("H", [1, 3])
def test_take(lens, n, counts, H):
    c, refs = a_cache(lens, H, 64, (max(lens) + n) // 64 + 2, spare=H * len(lens) * (n // 64 + 1) + 7, seed=n)
    check_take(c, refs, n, counts, "lens %s n %d" % (lens, n))


def test_take_beyond_the_table_and_strange_lengths():
    c, refs = a_cache([0, 0, 0], 2, 64, 3, spare=40)
    c["lens"].copy_(torch.tensor([190, 1 << 30, -5]))
    check_take(c, refs, 500, [500, -3, 1 << 30], "beyond the table")


@pytest.mark.parametrize("short", [0, 1, 5])
def test_take_all_or_none(short):
    c, refs = a_cache([60, 120, 0], 2, 64, 6, spare=2 * 6 - short)
    _, _, missing = check_take(c, refs, 128, None, "short of %d" % short)
    assert missing == short


def test_take_of_shared_and_strange_entries():
    c, refs = a_cache([300, 300, 300, 300], 2, 64, 8, spare=60, shared=0.5)
    pages = len(refs)
    c["table"][0, 0, 5], c["table"][1, 1, 5], c["table"][2, 0, 6] = pages, -7, c["table"][3, 0, 1]
    c["table"][3, 0, 5] = c["table"][3, 1, 5] = int((refs == 0).nonzero()[-1])
    refs = pg.count(c)
    c["lens"].copy_(torch.tensor([200, 130, 300, 300]))
    check_take(c, refs, 260, None, "shared")
    refs[5:15] = -3
    check_take(c, refs, 260, [260, 100, 1, 260], "negative counts")


@pytest.mark.parametrize("pages", [1023, 1024, 1025, 70_001])
def test_take_from_large_pools(pages):
    B, H, n = 6, 5, 64 * 40
    c, refs = a_cache([17] * B, H, 64, 45, spare=0, seed=pages)
    g = torch.Generator().manual_seed(pages)
    for name in ("k", "v", "bounds", "scales"):
        c[name] = torch.zeros((pages,) + c[name].shape[1:]).to(c[name].dtype)
    refs = (torch.rand(pages, generator=g) < 0.6).to(torch.int32)
    check_take(c, refs, n, [n, 64, 0, 1000, n, 47], "%d pages" % pages)


# ---- fork


def check_fork(c, refs, source, keep, what):
    say("fork", what)
    want, after = pg.fork(c, refs, source, keep)
    cache, r = on_gpu(c), refs.cuda()
    context().kv_fork(cache, r, torch.tensor(source, dtype=torch.int32, device="cuda"), keep=None if keep is None else torch.tensor(keep, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    same(cache, want, what)
    assert torch.equal(r.cpu(), after), what
    return want, after


@pytest.mark.parametrize("dtype,D,H", [(BF, 128, 2), (HF, 96, 3), (BF, 64, 1)])
@pytest.mark.parametrize("source", [[0, 1, 2, 3, 4], [0, 0, 0, 0, 0], [1, 2, 3, 4, 0], [4, 3, 2, 1, 0], [1, 1, 3, 3, -1], [-1, 5, 1 << 30, -7, 0], [2, 0, 2, 2, 3]])
def test_fork(dtype, D, H, source):
    for lens in ([0, 1, 64, 200, 63], [129, 135, 136, 137, 143], [640, 0, 700, 64, 191]):
        c, refs = a_cache(lens, H, D, 12, spare=9, seed=sum(lens), dtype=dtype, shared=0.3)
        check_fork(c, refs, source, None, "source %s lens %s" % (source, lens))


@pytest.mark.parametrize("keep", [[0, 0, 0, 0], [64, 65, 127, 128], [1 << 30] * 4, [-9, 63, 199, 200], [200, 201, 300, 640]])
@pytest.mark.parametrize("source", [[0, 1, 2, 3], [0, 0, 0, 0], [1, 0, 3, 2], [3, 3, 1, -1]])
def test_fork_of_first_tokens(source, keep):
    c, refs = a_cache([200, 641, 64, 300], 2, 64, 12, spare=9, seed=1, shared=0.3)
    check_fork(c, refs, source, keep, "source %s keep %s" % (source, keep))


def test_fork_releases_entries_behind_the_full_blocks():
    c, refs = a_cache([100, 300], 2, 64, 9, spare=60)
    table, refs, _ = pg.take(c, refs, 128)     # pages for blocks to come
    c["table"] = table
    _, after = check_fork(c, refs, [0, 0], None, "entries for blocks to come")
    assert (after[c["table"][1, 0, :6].long()] == 0).all() and (after[c["table"][0, 0, :1].long()] == 2).all()


def test_fork_twice_is_fork_of_fork():
    c, refs = a_cache([300, 80, 500], 2, 64, 9, spare=5)
    c, refs = check_fork(c, refs, [1, 2, 0], None, "first")
    c, refs = check_fork(c, refs, [0, 0, 1], None, "second")
    assert torch.equal(refs, pg.count(c))


# ---- free


@pytest.mark.parametrize("n", [0, 1, 255, 1024, 5001])
def test_free(n):
    say("free", n)
    g = torch.Generator().manual_seed(n)
    refs = torch.randint(0, 4, (300,), generator=g, dtype=torch.int32)
    pages = torch.randint(-50, 350, (n,), generator=g, dtype=torch.int32)
    r = refs.cuda()
    context().kv_free(r, pages.cuda())
    torch.cuda.synchronize()
    assert torch.equal(r.cpu(), pg.free(refs, pages))


# ---- compact


def check_compact(c, refs, what):
    say("compact", what)
    want, after, used = pg.compact(c, refs)
    ctx = context()
    for apart in (True, False):
        cache, r = on_gpu(c), refs.cuda()
        t_out, r_out = (torch.full_like(cache.table, 77), torch.full_like(r, 77)) if apart else (None, None)
        got = ctx.kv_compact(cache, r, table_out=t_out, refs_out=r_out)
        torch.cuda.synchronize()
        assert int(got) == used, what
        assert torch.equal((t_out if apart else cache.table).cpu(), want["table"]) and torch.equal((r_out if apart else r).cpu(), after), "%s apart %s" % (what, apart)
        same(cache, want, what, ("k", "v", "scales", "bounds", "tail_k", "tail_v", "lens", "evicted"))


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("lens,spare", [([0], 1), ([64], 0), ([64], 1), ([64], 40), ([200, 700, 0, 64], 3), ([200, 700, 0, 64], 500), ([1500] * 3, 30)])
def test_compact(D, lens, spare):
    c, refs = a_cache(lens, 2, D, max(lens) // 64 + 1, spare=spare, seed=spare, shared=0.3)
    check_compact(c, refs, "D %d lens %s spare %d" % (D, lens, spare))


def test_compact_leaves_entries_that_name_no_used_page():
    c, refs = a_cache([500, 300], 2, 64, 9, spare=40)
    pages = len(refs)
    c["table"][0, 0, 8], c["table"][0, 1, 8], c["table"][1, 0, 8] = pages, 1 << 30, pages - 1
    refs[pages - 1] = 0
    refs[3] = -2
    check_compact(c, refs, "strange entries")


def test_compact_of_a_compact_pool_changes_nothing():
    c, refs = a_cache([500, 300], 2, 64, 9, spare=40)
    c, refs, used = pg.compact(c, refs)
    assert (refs[:used] > 0).all()
    check_compact(c, refs, "compact already")


@pytest.mark.parametrize("pages", [2047, 2048, 5000])
def test_compact_over_several_chunks(pages):
    c, refs = a_cache([64 * 30] * 8, 4, 64, 31, spare=pages - 4 * 240, seed=pages)
    check_compact(c, refs, "%d pages" % pages)


# ---- packed appends


def starts_of(counts, first=0):
    at = [first]
    for n in counts:
        at.append(at[-1] + n)
    return at


@pytest.mark.parametrize("dtype,D,H", [(BF, 128, 2), (HF, 96, 3), (BF, 64, 1)])
@pytest.mark.parametrize("lens,counts", [([0], [1]), ([0, 63, 10], [1, 1, 0]), ([5, 0, 70, 64], [200, 64, 0, 131]), ([0] * 70, [b % 4 for b in range(70)]), ([63, 62, 1], [1, 2, 63])])
def test_append_packed_is_append(dtype, D, H, lens, counts):
    say("append packed", dtype, D, H, lens, counts)
    blocks = max(x + y for x, y in zip(lens, counts)) // 64 + 1
    g = torch.Generator().manual_seed(D + sum(counts))
    c = kv.new_cache(len(lens), H, D, blocks, dtype)
    most = max(lens)
    if most:
        kv.append(c, *(torch.randn(len(lens), most, H, D, generator=g).to(dtype) for _ in range(2)), torch.tensor(lens))
    c["lens"].copy_(torch.tensor(lens))
    c["evicted"].copy_(torch.randint(0, 2, (len(lens),), generator=g) * 0)
    before, behind = 3, 5
    starts = starts_of(counts, before)
    k, v = ((torch.randn(starts[-1] + behind, H, D, generator=g) * torch.exp2(torch.randint(-6, 7, (starts[-1] + behind, H, 1), generator=g))).to(dtype) for _ in range(2))
    padded = [torch.zeros(len(lens), max(counts), H, D, dtype=dtype) for _ in range(2)]
    for b, n in enumerate(counts):
        padded[0][b, :n], padded[1][b, :n] = k[starts[b] : starts[b] + n], v[starts[b] : starts[b] + n]
    st = torch.tensor(starts, dtype=torch.int32, device="cuda")
    ctx = context()
    # dense rows, and views of a projection that holds both
    fused = torch.cat([k, v], 1).cuda()
    dense, views = on_gpu(c), on_gpu(c)
    ctx.kv_append_packed(dense, k.cuda(), v.cuda(), st)
    ctx.kv_append_packed(views, fused[:, :H], fused[:, H:], st)
    kv.append(c, *padded, torch.tensor(counts))
    torch.cuda.synchronize()
    for cache in (dense, views):
        for name in ("k", "v", "scales", "bounds", "tail_k", "tail_v", "lens"):
            x, y = getattr(cache, name).cpu().float(), c[name].float()
            assert torch.equal(x, y), name


def test_append_packed_with_starts_outside_of_the_tokens():
    say("append packed: strange starts")
    k = torch.randn(100, 1, 64, generator=torch.Generator().manual_seed(0)).to(BF).cuda()
    ctx, c = context(), kv.new_cache(2, 1, 64, 4, BF)
    a, b = on_gpu(c), on_gpu(c)
    ctx.kv_append_packed(a, k, k, torch.tensor([-10, 70, 1 << 30], dtype=torch.int32, device="cuda"))
    ctx.kv_append_packed(b, k, k, torch.tensor([0, 70, 100], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    same(a, {name: getattr(b, name).cpu() for name in etf.KvCache.FIELDS}, "clamped")
    ctx.kv_append_packed(a, k, k, torch.tensor([50, 20, 20], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    same(a, {name: getattr(b, name).cpu() for name in etf.KvCache.FIELDS}, "no new tokens")


# ---- together


def test_served_from_packed_prompts_to_shared_pages():
    """Packed prompts into a pool, copies of sequences, single tokens of their own, an eviction, a sequence that leaves, the pool made
    compact: attention as over a cache of the same tokens in which every block has a page of its own from the start."""
    say("together")
    T, H, g, D, B, blocks = BF, 2, 3, 64, 4, 12
    gen = torch.Generator().manual_seed(11)
    ctx = context()
    rand = lambda *s: torch.randn(s, generator=gen).to(T).cuda()  # noqa: E731
    pool = etf.KvCache.alloc(B, H, D, blocks * 64, dtype=T, pages=60)
    refs = torch.zeros(60, dtype=torch.int32, device="cuda")
    plain = etf.KvCache.alloc(B, H, D, blocks * 64, dtype=T)
    counts = [200, 70, 0, 0]
    k, v, q = rand(270, H, D), rand(270, H, D), rand(270, H * g, D)
    starts = torch.tensor(starts_of(counts), dtype=torch.int32, device="cuda")
    cnt = torch.tensor(counts, dtype=torch.int32, device="cuda")
    out = ctx.prompt_attend(q, k, v, starts)
    assert int(ctx.kv_take(pool, refs, 200, counts=cnt)) == 0
    ctx.kv_append_packed(pool, k, v, starts)
    pool.lens += cnt
    # sequences 2 and 3: copies of 0, of 1's first whole block
    ctx.kv_fork(pool, refs, torch.tensor([0, 1, 0, 1], dtype=torch.int32, device="cuda"), keep=torch.tensor([1 << 20, 1 << 20, 1 << 20, 69], dtype=torch.int32, device="cuda"))
    for b, (s, n) in enumerate(((0, 200), (1, 70), (0, 200), (1, 64))):
        given = [x[int(starts[s]) : int(starts[s]) + n][None].expand(B, -1, -1, -1) for x in (k, v)]
        only = torch.zeros(B, dtype=torch.int32, device="cuda")
        only[b] = n
        ctx.kv_append(plain, *(x.contiguous() for x in given), counts=only)
        plain.lens += only
    assert torch.equal(pool.lens, plain.lens)
    # the last rows of the prompts' own attention, from exact keys, are near those over the cache's codes
    last = ctx.kv_attend(pool, torch.stack([q[199], q[269], q[199], q[263]])[:, None])
    assert torch.equal(last, ctx.kv_attend(plain, torch.stack([q[199], q[269], q[199], q[263]])[:, None]))
    assert (last[0, 0].float() - out[199].float()).abs().max() < 0.2     # e4m3 codes: 2^-4 of values around 1, averaged over many
    for step in range(130):
        k, v, q = rand(B, 1, H, D), rand(B, 1, H, D), rand(B, 1, H * g, D)
        assert int(ctx.kv_take(pool, refs)) == 0
        for cache in (pool, plain):
            ctx.kv_append(cache, k, v)
            cache.lens += 1
        if step % 40 == 0:
            assert torch.equal(ctx.kv_attend(pool, q), ctx.kv_attend(plain, q)), step
    used = int((refs > 0).sum())
    # an eviction by some weights takes the same blocks out of both
    mass = torch.rand(pool.table.shape, generator=gen).cuda()
    _, freed = ctx.kv_evict(pool, mass.clone(), 3, sink=1, recent=1)
    ctx.kv_free(refs, freed)
    ctx.kv_evict(plain, mass.clone(), 3, sink=1, recent=1)
    assert torch.equal(ctx.kv_attend(pool, q), ctx.kv_attend(plain, q))
    # sequence 1 leaves, sequence 3 becomes what 0 is; the pool is made compact
    source = torch.tensor([0, -1, 2, 0], dtype=torch.int32, device="cuda")
    ctx.kv_fork(pool, refs, source)
    want = ctx.kv_attend(plain, q[[0, 1, 2, 0]].contiguous())
    got = ctx.kv_attend(pool, q[[0, 1, 2, 0]].contiguous())
    assert torch.equal(got[[0, 2]], want[[0, 2]]) and torch.equal(got[3], got[0]) and (got[1] == 0).all()
    left = int(ctx.kv_compact(pool, refs))
    assert left < used and (refs[:left] > 0).all() and (refs[left:] == 0).all() and int(pool.table.max()) < left
    c = {name: getattr(pool, name).cpu() for name in etf.KvCache.FIELDS}
    assert torch.equal(pg.count(c), refs.cpu())
    assert torch.equal(ctx.kv_attend(pool, q[[0, 1, 2, 0]].contiguous()), got)
    pool.k[left:].view(torch.uint8).fill_(0x7F)     # nothing reads what lies behind
    pool.v[left:].view(torch.uint8).fill_(0x7F)
    assert torch.equal(ctx.kv_attend(pool, q[[0, 1, 2, 0]].contiguous()), got)


def test_a_draft_is_taken_back_after_a_fork():
    """A block that others share already is completed again: it gets another page, and theirs stays as it is."""
    say("draft after a fork")
    T, H, D = BF, 2, 64
    gen = torch.Generator().manual_seed(12)
    ctx = context()
    rand = lambda n: torch.randn(2, n, H, D, generator=gen).to(T).cuda()  # noqa: E731
    pool = etf.KvCache.alloc(2, H, D, 256, dtype=T, pages=8)
    refs = torch.zeros(8, dtype=torch.int32, device="cuda")
    only = torch.tensor([60, 0], dtype=torch.int32, device="cuda")
    ctx.kv_append(pool, rand(60), rand(60), counts=only)
    pool.lens += only
    draft = torch.tensor([10, 0], dtype=torch.int32, device="cuda")
    assert int(ctx.kv_take(pool, refs, 10, counts=draft)) == 0
    ctx.kv_append(pool, rand(10), rand(10), counts=draft)
    pool.lens += draft
    ctx.kv_fork(pool, refs, torch.tensor([0, 0], dtype=torch.int32, device="cuda"))
    q = torch.randn(2, 1, 2 * H, D, generator=gen).to(T).cuda()
    before = ctx.kv_attend(pool, q[[0, 0]].contiguous())
    assert torch.equal(before[0], before[1]) and pool.lens.tolist() == [70, 70]
    page = pool.table[1, :, 0].clone()
    assert torch.equal(pool.table[0, :, 0], page) and (refs[page.long()] == 2).all()
    # two of the ten were right; four others follow
    pool.lens[0] -= 8
    more = torch.tensor([4, 0], dtype=torch.int32, device="cuda")
    assert int(ctx.kv_take(pool, refs, 4, counts=more)) == 0
    assert (pool.table[0, :, 0] != page).all() and torch.equal(pool.table[1, :, 0], page) and (refs[page.long()] == 1).all()
    ctx.kv_append(pool, rand(4), rand(4), counts=more)
    pool.lens += more
    after = ctx.kv_attend(pool, q[[0, 0]].contiguous())
    assert pool.lens.tolist() == [66, 70] and torch.equal(after[1], before[1]) and not torch.equal(after[0], before[0])


def test_pools_of_more_than_4_gib():
    """Offsets of pages beyond 2^32 bytes."""
    say("large pool")
    pages, D = 540_000, 128     # 4.4 GB of keys
    assert pages * 64 * D > 1 << 32
    pool = etf.KvCache.alloc(1, 1, D, 64 * 3, pages=pages)
    for i, p in enumerate((pages - 1, pages - 7)):
        pool.k[p].view(torch.uint8).fill_(17 + i)
        pool.v[p].view(torch.uint8).fill_(33 + i)
        pool.bounds[p].view(torch.uint8).fill_(49 + i)
        pool.scales[p].fill_(2.0 ** i)
        pool.table[0, 0, i] = p
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[pool.table[0, 0, :2].long()] = 1
    ctx = context()
    pool.lens.fill_(130)
    assert int(ctx.kv_take(pool, refs, 64)) == 0 and pool.table.tolist() == [[[pages - 1, pages - 7, 0]]]
    used = ctx.kv_compact(pool, refs)
    assert int(used) == 3 and pool.table.tolist() == [[[1, 2, 0]]] and refs[:4].tolist() == [1, 1, 1, 0] and int(refs.sum()) == 3
    for i, p in enumerate((1, 2)):
        assert (pool.k[p].view(torch.uint8) == 17 + i).all() and (pool.v[p].view(torch.uint8) == 33 + i).all() and (pool.bounds[p].view(torch.uint8) == 49 + i).all()
        assert (pool.scales[p] == 2.0 ** i).all()


def test_calls_on_another_stream_than_the_current_one():
    say("another stream")
    c, refs = a_cache([63, 130, 191, 0], 2, 64, 9, spare=60, shared=0.3)
    want, after = pg.fork(c, refs, [1, 1, 0, 2])
    table, after, lack = pg.take(want, after, 70)
    want, after, many = pg.compact(dict(want, table=table), after)
    ctx, cache, r = context(), on_gpu(c), refs.cuda()
    src = torch.tensor([1, 1, 0, 2], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        ctx.kv_fork(cache, r, src)
        missing = ctx.kv_take(cache, r, 70)
        used = ctx.kv_compact(cache, r)
    torch.cuda.synchronize()
    same(cache, want, "another stream")
    assert torch.equal(r.cpu(), after) and int(missing) == lack and int(used) == many


def test_in_a_graph():
    """A step's calls captured and replayed, with eager calls on the same arrays between the replays."""
    say("graph")
    c, refs0 = a_cache([63, 130, 191, 0], 2, 64, 9, spare=60, shared=0.3)
    source = [1, 1, 0, 2]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = etf.Context(device=0, stream=side.cuda_stream)
        cache, refs = on_gpu(c), refs0.cuda()
        src = torch.tensor(source, dtype=torch.int32, device="cuda")
        missing, used = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
        room = {name: torch.empty(size(cache) + 256, dtype=torch.uint8, device="cuda") for name, size in
                (("take", lambda x: ctx.kv_take_workspace_bytes(x, 70)), ("fork", ctx.kv_fork_workspace_bytes), ("compact", ctx.kv_compact_workspace_bytes))}

        def step():
            ctx.kv_fork(cache, refs, src, ws=room["fork"])
            ctx.kv_take(cache, refs, 70, missing=missing, ws=room["take"])
            ctx.kv_compact(cache, refs, used=used, ws=room["compact"])

        def restore(oracle):
            for name in etf.KvCache.FIELDS:
                getattr(cache, name).copy_(oracle[name])
            refs.copy_(refs0)

        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        want, r = pg.fork(c, refs0, source)
        table, r, lack = pg.take(want, r, 70)
        want, r, many = pg.compact(dict(want, table=table), r)
        for i in range(3):
            restore(c)
            graph.replay()
            side.synchronize()
            same(cache, want, "replay %d" % i)
            assert torch.equal(refs.cpu(), r) and int(missing) == lack and int(used) == many
            restore(c)
            step()
            side.synchronize()
            same(cache, want, "eager %d" % i)


def test_append_packed_and_free_on_another_stream_and_in_a_graph():
    """Captured and replayed, with eager calls on the same arrays between the replays; the shares of pages that are listed more than once."""
    say("append packed, free: streams, graph")
    T, H, D, lens, counts = HF, 2, 96, [60, 0, 130], [70, 64, 3]
    gen = torch.Generator().manual_seed(31)
    c = kv.new_cache(3, H, D, 4, T)
    kv.append(c, *(torch.randn(3, 130, H, D, generator=gen).to(T) for _ in range(2)), torch.tensor(lens))
    c["lens"].copy_(torch.tensor(lens))
    starts = starts_of(counts)
    k, v = (torch.randn(starts[-1], H, D, generator=gen).to(T) for _ in range(2))
    padded = [torch.zeros(3, 70, H, D, dtype=T) for _ in range(2)]
    for b, n in enumerate(counts):
        padded[0][b, :n], padded[1][b, :n] = k[starts[b] : starts[b] + n], v[starts[b] : starts[b] + n]
    before = {name: c[name].clone() for name in etf.KvCache.FIELDS}
    kv.append(c, *padded, torch.tensor(counts))
    refs0 = torch.tensor([3, 1, 0, 2, 5], dtype=torch.int32)
    listed = torch.tensor([0, 0, -1, 1, 1, 2, 3, 9, 4, 0, 0], dtype=torch.int32)
    want = torch.tensor([0, 0, 0, 1, 4], dtype=torch.int32)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        kg, vg, st, lg, refs = k.cuda(), v.cuda(), torch.tensor(starts, dtype=torch.int32, device="cuda"), listed.cuda(), refs0.cuda()
        cache = on_gpu(before)
        ctx = etf.Context(device=0, stream=side.cuda_stream)
        side.synchronize()

        def step():
            ctx.kv_append_packed(cache, kg, vg, st)
            ctx.kv_free(refs, lg)

        def restore():
            for name in etf.KvCache.FIELDS:
                getattr(cache, name).copy_(before[name])
            refs.copy_(refs0)

        def right(what):
            side.synchronize()
            for name in etf.KvCache.FIELDS:
                x, y = getattr(cache, name).cpu().float(), c[name].float()
                assert torch.equal(x, y), "%s: %s" % (what, name)
            assert torch.equal(refs.cpu(), want), what

        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        for i in range(3):
            restore()
            graph.replay()
            right("replay %d" % i)
            restore()
            step()
            right("eager %d" % i)
        restore()
    side.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        step()
    right("another current stream")


def test_append_packed_of_tokens_beyond_2_to_the_32():
    """Keys and values that lie beyond 2^32 elements, of tokens of which most are no sequence's."""
    say("append packed: far tokens")
    H, D = 8, 128
    tokens = (1 << 32) // (H * D) + 4321
    k = torch.zeros(tokens, H, D, dtype=BF, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(5)
    k[-300:] = torch.randn(300, H, D, generator=gen, device="cuda").to(BF)
    assert (tokens - 300) * H * D > 1 << 32
    ctx = context()
    far, near = (etf.KvCache.alloc(3, H, D, 256, dtype=BF) for _ in range(2))
    starts = torch.tensor([0, 130, 130, 300], dtype=torch.int32, device="cuda")
    ctx.kv_append_packed(far, k, k, starts + (tokens - 300))
    few = k[-300:].clone()
    ctx.kv_append_packed(near, few, few, starts)
    torch.cuda.synchronize()
    full = torch.tensor([2, 0, 2])
    for b in range(3):
        n = int(full[b])
        for h in range(H):
            for p in near.table[b, h, :n].tolist():
                for name in ("k", "v", "bounds"):
                    assert torch.equal(getattr(far, name)[p].view(torch.uint8), getattr(near, name)[p].view(torch.uint8)), (b, h, name)
                assert torch.equal(far.scales[p], near.scales[p])
    same_open = [torch.equal(far.tail_k[b, :, 0, : m], near.tail_k[b, :, 0, : m]) and torch.equal(far.tail_v[b, :, 0, :, : m], near.tail_v[b, :, 0, :, : m]) for b, m in ((0, 2), (2, 42))]
    assert all(same_open)
    assert torch.equal(near.tail_k[2, :, 0, :42].transpose(0, 1), few[258:]) and torch.equal(near.tail_k[0, :, 0, :2].transpose(0, 1), few[128:130])


def test_example_of_shared_prompts():
    say("example")
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "shared_prompts.py")
    spec = importlib.util.spec_from_file_location("shared_prompts", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    for args in (["--batch", "6", "--heads", "2", "--shared", "333", "--own", "90", "--tokens", "70", "--head-dim", "64"], ["--batch", "1", "--heads", "1", "--group", "3", "--shared", "64", "--own", "1", "--tokens", "1"]):
        cache, refs, used, off = example.main(args)
        # off by the roundings of bf16 only: those of the weights and of the output
        most = float(cache.tail_v.abs().max().clamp_min(448 * cache.scales[:, 1].max()))
        assert off <= 2 * 2.0 ** -8 * most + 2.0 ** -12 * most
        c = {name: getattr(cache, name).cpu() for name in etf.KvCache.FIELDS}
        assert torch.equal(pg.count(c), refs.cpu()) and (refs[:used] > 0).all() and not refs[used:].any()
