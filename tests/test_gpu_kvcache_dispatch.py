"""Both sides of every size at which the cache calls change their kernel or its launch, against the oracle in float64; bounds as in test_gpu_kvcache.py."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import kvcache as kv  # noqa: E402
import paper_1509_05186_amd as etf  # noqa: E402

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_gpu_kvcache import BF, HF, bounds_only, check_out, context, filled, on_gpu, queries, say  # noqa: E402

INF = math.inf


def attend(c, q, scale, counts=None, lists=None):
    """kv.attend with a matrix product for each (sequence, head) instead of a loop over rows."""
    B, n, Hq, D = q.shape
    H, blocks = c["table"].shape[1:]
    g, z = Hq // H, lambda *s: torch.zeros(*s, dtype=torch.float64)  # noqa: E731
    r = dict(out=z(B, n, Hq, D), lse=torch.full((B, n, Hq), -INF).double(), mass=z(B, H, blocks), size=z(B, n, Hq, D), reach=z(B, n, Hq),
             mag=z(B, n, Hq), seen=z(B, n, Hq), vmax=z(B, n, Hq))
    for b in range(B):
        count = n if counts is None else min(max(int(counts[b]), 0), n)
        if count == 0:
            continue
        length = kv._len(c, b)
        vis = (length - count + 1 + torch.arange(count)).clamp(min=0)
        for h in range(H):
            k, v, there = kv.tokens(c, b, h)
            if len(k) == 0:
                continue
            at = torch.arange(len(k))
            see = (at < vis[:, None]) & there
            if lists is not None:
                whole = vis // 64
                named = torch.zeros(count, blocks + 1, dtype=torch.bool)
                rows = lists[b, :count, h].long()
                ok = (rows >= 0) & (rows < whole[:, None])
                named.scatter_(1, torch.where(ok, rows, blocks), True)
                see &= (at // 64 >= whole[:, None]) | named[:, (at // 64).clamp(max=blocks)]
            see = see[:, None].expand(count, g, len(k))
            qq = q[b, :count, h * g : h * g + g].double()
            s = (qq @ k.T * scale).masked_fill(~see, -INF)
            lse = torch.logsumexp(s, -1)
            p = torch.exp(s - torch.where(lse == -INF, 0.0, lse)[..., None])
            sl = (b, slice(0, count), slice(h * g, h * g + g))
            r["out"][sl], r["lse"][sl], r["size"][sl] = p @ v, lse, p @ v.abs()
            r["reach"][sl] = torch.where(see, s.abs(), 0.0).amax(-1)
            r["mag"][sl] = torch.where(see, qq.abs() @ k.abs().T * scale, 0.0).amax(-1)
            r["seen"][sl] = see.sum(-1).double()
            r["vmax"][sl] = torch.where(see, v.abs().amax(1), 0.0).amax(-1)
            r["mass"][b, h] += torch.nn.functional.pad(p.sum((0, 1)), (0, (blocks + 1) * 64 - len(k))).view(-1, 64).sum(1)[:blocks]
    return r


def test_the_products_are_the_oracles_loop():
    c, rand = filled(BF, 64, 2, [300, 70, 0], seed=1)
    c["table"][0, 1, 2] = -1
    q, counts = queries(rand, BF, 3, 3, 6, 64), torch.tensor([3, 2, 1])
    lists = torch.tensor([0, 3, -1, 99], dtype=torch.int32).expand(3, 3, 2, 4)
    for some in (None, lists):
        x, y = attend(c, q, 0.125, counts, some), kv.attend(c, q, 0.125, counts, some)
        for name in x:
            torch.testing.assert_close(x[name], y[name], rtol=1e-12, atol=1e-12)


# (sequence, token, head, tile of 16 heads) units: 2048 and more go one to a wave.  Numbers of a head's units that four does not divide; counts
# that leave some to padding
@pytest.mark.parametrize("dtype,D,H,g,n,lens,counts,units", [
    (BF, 96, 3, 5, 227, [300, 500, 227], None, 2043),
    (BF, 96, 3, 5, 228, [300, 500, 228], [228, 100, 3], 2052),
    (HF, 96, 3, 5, 230, [300, 500, 230], None, 2070),
    (HF, 64, 2, 17, 257, [400, 257], [257, 130], 2056),
    (BF, 128, 1, 40, 341, [341, 500], None, 2046),
    (BF, 128, 1, 40, 342, [342, 500], [1, 342], 2052),
])
def test_listed_units_few_and_many(dtype, D, H, g, n, lens, counts, units):
    say("listed units", dtype, D, H, g, n, lens, counts)
    B = len(lens)
    assert B * n * H * -(-g // 16) == units
    c, rand = filled(dtype, D, H, lens, seed=n, evicted=[b % 2 for b in range(B)])
    c["table"][0, 0, 1] = -1
    q = queries(rand, dtype, B, n, H * g, D)
    cnt = None if counts is None else torch.tensor(counts, dtype=torch.int32)
    lists = torch.stack([torch.randperm(9, generator=rand)[:5] - 1 for _ in range(B * n * H)]).to(torch.int32).view(B, n, H, 5)     # -1 and blocks past the end among them
    lse = torch.full(q.shape[:3], 7.0, device="cuda")
    out = context().kv_attend(on_gpu(c), q.cuda(), counts=None if cnt is None else cnt.cuda(), lists=lists.cuda(), lse=lse, out=torch.full_like(q, 5.0, device="cuda"))
    check_out(attend(c, q, D ** -0.5, cnt, lists), out, dtype, "listed", lse)


# tables so wide that a wave of the scores goes through several tiles of tokens, counts that end inside such a turn, at its end and before its start
@pytest.mark.parametrize("dtype,D,g,n,counts,turns", [(BF, 64, 16, 37, 29, 4), (HF, 96, 16, 37, 28, 4), (BF, 128, 3, 150, 101, 4), (BF, 64, 20, 80, 80, 8), (HF, 64, 1, 300, 1, 2), (BF, 64, 16, 15, 15, 1)])
def test_scores_of_several_tiles_to_a_wave(dtype, D, g, n, counts, turns):
    say("turns", dtype, D, g, n, counts)
    blocks, whole = 8192, 30
    tokens = 16 // min(16, 1 << (g - 1).bit_length())
    assert max(1, min(8, blocks // 64 * -(-n // tokens) // 1024)) == turns
    c, rand = bounds_only(D, blocks, whole, 40, g + n, dtype=dtype)
    q = queries(rand, dtype, 1, n, g, D)
    cnt = torch.tensor([counts], dtype=torch.int32)
    lists = context().kv_select(on_gpu(c), q.cuda(), 6, sink=1, recent=1, counts=cnt.cuda())
    assert torch.equal(lists.cpu(), kv.select(c, q, 6, 1, 1, cnt))


def many_sequences(dtype, D, H, lens, long, blocks, seed):
    """Sequences of a few tokens and one long one in a wide table, with pages for what is there only."""
    g = torch.Generator().manual_seed(seed)
    B, short = len(lens), max(lens)
    own = [x // 64 for x in lens]
    own[long[0]] = long[1] // 64
    table, page = torch.full((B, H, blocks), -1, dtype=torch.int32), 0
    for b in range(B):
        for h in range(H):
            table[b, h, : own[b]] = torch.arange(page, page + own[b])
            page += own[b]
    c = kv.new_cache(B, H, D, blocks, dtype, pages=max(1, page), table=table)
    counts = torch.tensor(lens)
    counts[long[0]] = 0
    kv.append(c, *(torch.randn(B, short, H, D, generator=g).to(dtype) for _ in range(2)), counts)
    one = torch.zeros(B, dtype=torch.int64)
    one[long[0]] = long[1]
    kv.append(c, *(torch.randn(1, long[1], H, D, generator=g).to(dtype).expand(B, -1, -1, -1) for _ in range(2)), one)
    c["lens"].copy_(counts + one)
    return c, g


# prompts: 1024 (sequence, head, tile of 128 rows) units and more are not cut into ranges
@pytest.mark.parametrize("dtype,D,H,g,n,B,units", [(BF, 64, 16, 1, 70, 63, 1008), (BF, 64, 16, 1, 70, 64, 1024), (HF, 96, 8, 2, 65, 64, 1024), (HF, 128, 31, 1, 129, 17, 1054)])
def test_prompts_of_few_and_many_units(dtype, D, H, g, n, B, units):
    say("prompts", dtype, D, H, g, n, B)
    assert B * H * -(-n * g // 128) == units
    lens = [n + (b * 13) % 60 for b in range(B)]
    c, rand = many_sequences(dtype, D, H, lens, (5, 700), 12, units)
    q = queries(rand, dtype, B, n, H * g, D)
    cnt = torch.tensor([n if b % 7 else b % n for b in range(B)], dtype=torch.int32)
    lse, mass = torch.full(q.shape[:3], 7.0, device="cuda"), torch.empty(c["table"].shape, device="cuda")
    want, cache = attend(c, q, D ** -0.5, cnt), on_gpu(c)
    check_out(want, context().kv_attend(cache, q.cuda(), counts=cnt.cuda(), lse=lse), dtype, "prompts", lse)
    check_out(want, context().kv_attend(cache, q.cuda(), counts=cnt.cuda(), lse=lse, mass_out=mass), dtype, "prompts, weights", lse, mass)


# single tokens: more units than a round of workgroups holds, than two and than three; tables around the width from which on they are cut into ranges
@pytest.mark.parametrize("dtype,D,H,B,blocks", [(BF, 64, 8, 64, 33), (BF, 64, 8, 70, 33), (HF, 64, 8, 130, 33), (BF, 96, 8, 200, 33), (HF, 128, 8, 200, 32), (BF, 64, 1, 100, 16), (BF, 64, 1, 100, 17), (BF, 64, 2, 64, 32),
                                               (HF, 64, 2, 64, 33)])
def test_tokens_of_few_and_many_units(dtype, D, H, B, blocks):
    say("tokens", dtype, D, H, B, blocks)
    lens = [1 + (b * 29) % 150 for b in range(B)]
    c, rand = many_sequences(dtype, D, H, lens, (B // 2, 64 * blocks - 3), blocks, B)
    q = queries(rand, dtype, B, 1, 3 * H, D)
    cnt = torch.tensor([0 if b % 11 == 3 else 1 for b in range(B)], dtype=torch.int32)
    lse, mass = torch.full(q.shape[:3], 7.0, device="cuda"), torch.empty(c["table"].shape, device="cuda")
    want, cache = attend(c, q, D ** -0.5, cnt), on_gpu(c)
    check_out(want, context().kv_attend(cache, q.cuda(), counts=cnt.cuda(), lse=lse), dtype, "tokens", lse)
    check_out(want, context().kv_attend(cache, q.cuda(), counts=cnt.cuda(), lse=lse, mass_out=mass), dtype, "tokens, weights", lse, mass)
