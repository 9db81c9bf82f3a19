"""Appends, pages taken, forks, evictions, drafts taken back and pools made compact, in random order: after every call the cache, the shares and what the
call returns are the oracle's, and shares and entries agree."""
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import kvcache as kv, pages as pg  # noqa: E402
import paper_1509_05186_amd as etf  # noqa: E402

BF, HF = torch.bfloat16, torch.float16


def say(*a):
    print(*a, flush=True)


def bits(t):
    t = t.cpu().contiguous()
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t.view(torch.int16) if t.element_size() == 2 else t.view(torch.int32)


def same(cache, c, what):
    for name in etf.KvCache.FIELDS:
        x, y = getattr(cache, name).cpu(), c[name]
        if name in ("k", "v", "bounds"):     # a zero is one with either sign
            assert torch.equal(x.float(), y.float()), "%s: %s" % (what, name)
        else:
            assert torch.equal(bits(x), bits(y)), "%s: %s" % (what, name)


@pytest.mark.parametrize("seed", range(16))
def test_random_flows(seed):
    rng, gen = random.Random(seed), torch.Generator().manual_seed(seed)
    dtype, D = rng.choice([BF, HF]), rng.choice([64, 96, 128])
    B, H, blocks = rng.choice([1, 3, 6]), rng.choice([1, 2]), rng.choice([4, 9])
    pages = B * H * blocks * rng.choice([1, 2]) // rng.choice([1, 2]) + 1
    c = kv.new_cache(B, H, D, blocks, dtype, pages=pages, table=torch.full((B, H, blocks), -1))
    refs = torch.zeros(pages, dtype=torch.int32)
    cache = etf.KvCache(**{name: c[name].cuda() for name in etf.KvCache.FIELDS})
    r = refs.cuda()
    ctx = etf.Context(device=0, stream=torch.cuda.current_stream().cuda_stream)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    say("flow", seed, dtype, "B %d H %d D %d blocks %d pages %d" % (B, H, D, blocks, pages))
    before = [None] * B  # what lens was before the last append, where it may go back to that
    for step in range(40):
        what = rng.choice(["append", "append", "append", "fork", "evict", "compact", "back", "ahead"])
        if what in ("append", "ahead"):
            n = rng.choice([1, 1, 3, 17, 64, 100, 190])
            counts = [rng.choice([0, n, n, rng.randrange(n + 1)]) for _ in range(B)]
            if what == "append" and rng.random() < 0.2:
                counts = None
            table, after, missing = pg.take(c, refs, n, counts)
            lack = ctx.kv_take(cache, r, n, counts=None if counts is None else ints(counts))
            c["table"], refs = table, after
            assert int(lack) == missing, step
            if what == "append" and missing == 0:
                each = counts or [n] * B
                lens = c["lens"].tolist()
                k, v = (torch.randn(B, n, H, D, generator=gen).to(dtype) for _ in range(2))
                if rng.random() < 0.5:
                    ctx.kv_append(cache, k.cuda(), v.cuda(), counts=ints(each))
                else:
                    lie = lambda x: torch.cat([x[b, :m] for b, m in enumerate(each)] + [x[0, :1]]).cuda()  # noqa: E731
                    ctx.kv_append_packed(cache, lie(k), lie(v), ints([sum(each[:b]) for b in range(B + 1)]))
                kv.append(c, k, v, torch.tensor(each))
                most = blocks * 64 + 63
                for b in range(B):
                    now = min(lens[b] + each[b], most)
                    if each[b]:
                        before[b] = lens[b] if now // 64 - lens[b] // 64 <= 1 else None
                    c["lens"][b] = now
                cache.lens.copy_(c["lens"])
        elif what == "back":
            for b in range(B):
                if before[b] is not None and rng.random() < 0.5:
                    c["lens"][b] = before[b]
                before[b] = None
            cache.lens.copy_(c["lens"])
        elif what == "fork":
            source = [rng.choice([b, b, rng.randrange(-1, B)]) for b in range(B)]
            keep = [rng.choice([0, 64, 100, 200, 1 << 20]) for _ in range(B)] if rng.random() < 0.5 else None
            ctx.kv_fork(cache, r, ints(source), keep=None if keep is None else ints(keep))
            c, refs = pg.fork(c, refs, source, keep)
            before = [None] * B
        elif what == "evict":
            budget = rng.choice([1, 2, 5, 20])
            mass = torch.rand(B, H, blocks, generator=gen)
            kept, freed = ctx.kv_evict(cache, mass.cuda(), budget, recent=min(1, budget), ahead=True)
            c["table"], c["lens"], c["evicted"], out, gone = pg.evict(c, mass, budget, 0, min(1, budget))
            assert torch.equal(kept.cpu(), out) and torch.equal(freed.cpu(), gone), step
            ctx.kv_free(r, freed)
            refs = pg.free(refs, gone)
            before = [None] * B
        else:
            used = ctx.kv_compact(cache, r)
            c, refs, many = pg.compact(c, refs)
            assert int(used) == many, step
        torch.cuda.synchronize()
        same(cache, c, "step %d %s" % (step, what))
        assert torch.equal(r.cpu(), refs) and torch.equal(pg.count(c), refs), "step %d %s" % (step, what)
