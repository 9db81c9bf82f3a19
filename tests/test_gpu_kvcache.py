"""Attention over a cache in 8 bits on the GPU against the oracle in float64 (oracle/kvcache.py).

Bounds.  With u the type's rounding (half its epsilon) and e = 2^-24: a logit is a sum of D products that are exact in float32, so
it is off by at most delta = (D + 4) e mag, mag = sum_d |q_d k_d| scale; its exponential by 2 delta + 4 e (1 + reach).  A weight is
then rounded to the type (u), and sums of `seen` terms in float32 add seen * e of their absolute terms.  With size = sum p |v| that
makes out off by (u + 2 w) size + u |out|, w = 2 delta + 4 e (1 + reach) + seen e.  In float16 a weight below the type's normal
numbers is off by 2^-25 of the largest (seen 2^-25 vmax in all), a value, taken at half its size, by 2^-24, the output by 2^-25.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import kvcache as kv  # noqa: E402
import paper_1509_05186_amd as etf  # noqa: E402

BF, HF = torch.bfloat16, torch.float16
E = 2.0 ** -24


def say(*a):
    print(*a, flush=True)


def context():
    return etf.Context(device=0, stream=torch.cuda.current_stream().cuda_stream)


def on_gpu(c):
    return etf.KvCache(**{name: c[name].cuda() for name in etf.KvCache.FIELDS})


def filled(dtype, D, H, lens, blocks=None, seed=0, evicted=None, scatter=True):
    """An oracle's cache with these lengths, made by the oracle; pages in random order, unwritten places not a number."""
    g = torch.Generator().manual_seed(seed)
    B = len(lens)
    blocks = max(lens) // 64 + 1 if blocks is None else blocks
    table = (torch.randperm(B * H * blocks + 5, generator=g)[: B * H * blocks] if scatter else torch.arange(B * H * blocks)).view(B, H, blocks)
    c = kv.new_cache(B, H, D, blocks, dtype, pages=B * H * blocks + 5, table=table)
    c["tail_k"].fill_(math.nan)
    c["tail_v"].fill_(math.nan)
    for name in ("k", "v", "bounds"):
        c[name].copy_(torch.full(c[name].shape, math.nan).to(torch.float8_e4m3fn))
    c["scales"].fill_(math.nan)
    if evicted is not None:
        c["evicted"].copy_(torch.tensor(evicted))
    n = max(lens)
    if n:
        shift = torch.randn(B, n // 32 + 1, H, D, generator=g).repeat_interleave(32, 1)[:, :n]
        k = (torch.randn(B, n, H, D, generator=g) + shift).to(dtype)
        v = (torch.randn(B, n, H, D, generator=g) * torch.exp(torch.randn(B, 1, H, 1, generator=g))).to(dtype)
        kv.append(c, k, v, torch.tensor(lens))
    c["lens"].copy_(torch.tensor(lens))
    return c, g


def queries(g, dtype, B, n, Hq, D, size=1.0):
    return (size * torch.randn(B, n, Hq, D, generator=g)).to(dtype)


def check_out(r, out, dtype, what, lse=None, mass=None, rows=1):
    u, D = torch.finfo(dtype).eps / 2, out.shape[-1]
    delta = (D + 4) * E * r["mag"]
    p = 2 * delta + 4 * E * (1 + r["reach"])
    w = (p + r["seen"] * E)[..., None]
    tol = (u + 2 * w) * r["size"] + u * r["out"].abs() + 1e-30
    if dtype == HF:
        tol += 2.0 ** -25 * r["seen"][..., None] * r["vmax"][..., None] + 2.0 ** -24 + 2.0 ** -25
    out, some = out.double().cpu(), ~torch.isnan(r["out"])   # what is not a number has to be none here either
    assert torch.equal(some, ~torch.isnan(out)), what
    off, tol = (out - r["out"]).abs()[some], tol[some]
    assert (off <= tol).all(), "%s: out %.3g over its bound" % (what, float((off / tol).max()))
    if lse is not None:
        lse = lse.double().cpu()
        none, some = r["lse"] == -math.inf, torch.isfinite(r["lse"])
        assert torch.equal(none, lse == -math.inf) and torch.equal(torch.isnan(r["lse"]), torch.isnan(lse)), what
        off = (lse - r["lse"]).abs()[some]
        tol = (p + r["seen"] * E + 4 * E * (1 + r["lse"].abs()))[some]
        assert (off <= tol).all(), "%s: lse %.3g over its bound" % (what, float((off / tol).max()))
    if mass is not None:
        worst = float((2 * p + 2 * r["seen"] * E + 8 * E * (1 + r["reach"])).max()) + 4 * E
        off = (mass.double().cpu() - r["mass"]).abs()
        assert (off <= worst * r["mass"] + 1e-30).all(), "%s: mass" % what


def same_cache(got, want, what, before=None):
    for name in etf.KvCache.FIELDS:
        x, y = getattr(got, name).cpu(), want[name]
        if x.dtype == torch.float8_e4m3fn:
            x, y = x.float(), y.float()
        ok = (x == y) | (torch.isnan(x.float()) & torch.isnan(y.float()))
        assert ok.all(), "%s: %s differs in %d places" % (what, name, int((~ok).sum()))


# ---- append


@pytest.mark.parametrize("dtype,D,H", [(BF, 128, 2), (HF, 96, 3), (BF, 64, 1), (HF, 128, 1)])
@pytest.mark.parametrize("lens,n,counts", [([0, 0], 1, None), ([0, 63], 1, None), ([62, 127, 64], 3, [3, 0, 2]), ([0, 64, 5], 64, None), ([1, 30], 200, [200, 131]),
                                           ([63], 65, None), ([10], 182, None)])
def test_append(dtype, D, H, lens, n, counts):
    say("append", dtype, D, H, lens, n, counts)
    blocks = (max(lens) + n) // 64 + 1
    c, g = filled(dtype, D, H, lens, blocks=blocks, seed=n, evicted=[i % 2 for i in range(len(lens))])
    k, v = (torch.randn(len(lens), n, H, D, generator=g) * torch.exp2(torch.randint(-6, 7, (len(lens), n, H, 1), generator=g)) for _ in range(2))
    k, v = k.to(dtype), v.to(dtype)
    k[0, 0] = 0
    cnt = None if counts is None else torch.tensor(counts, dtype=torch.int32)
    cache = on_gpu(c)
    context().kv_append(cache, k.cuda(), v.cuda(), counts=None if cnt is None else cnt.cuda())
    kv.append(c, k, v, cnt)
    same_cache(cache, c, "append")


def test_append_token_by_token_is_append_at_once():
    say("append token by token")
    ctx, T, D, H = context(), BF, 64, 2
    g = torch.Generator().manual_seed(9)
    k, v = (torch.randn(1, 135, H, D, generator=g).to(T).cuda() for _ in range(2))
    caches = []
    for piece in (1, 50, 135):
        cache = etf.KvCache.alloc(1, H, D, 135, dtype=T)
        for i in range(0, 135, piece):
            ctx.kv_append(cache, k[:, i : i + piece], v[:, i : i + piece])
            cache.lens += min(piece, 135 - i)
        caches.append(cache)
    q = torch.randn(1, 1, 4, D, generator=g).to(T).cuda()
    outs = [ctx.kv_attend(x, q) for x in caches]
    for cache, out in zip(caches[1:], outs[1:]):
        assert torch.equal(cache.k.float()[:4], caches[0].k.float()[:4]) and torch.equal(cache.v.float()[:4], caches[0].v.float()[:4])
        assert torch.equal(out, outs[0])


@pytest.mark.parametrize("dtype", [BF, HF])
def test_append_extremes(dtype):
    """Zeros, the type's largest and smallest numbers, infinities and what is not a number, full blocks and open ones."""
    say("append extremes", dtype)
    D, H, n = 64, 1, 64 * 5 + 9
    g = torch.Generator().manual_seed(10)
    k, v = (torch.randn(1, n, H, D, generator=g).to(dtype) for _ in range(2))
    info = torch.finfo(dtype)
    k[0, :64], v[0, :64] = 0, -0.0
    k[0, 64:128] *= info.max / 8
    v[0, 64:128] *= info.smallest_normal
    k[0, 130, 0, 3], v[0, 140, 0, 60], k[0, 141, 0, 0] = math.inf, math.nan, -math.inf
    k[0, 192:256], v[0, 192:256] = math.nan, 1.0       # a block without a finite token
    k[0, 256, 0], v[0, 256, 0] = info.max, -info.max
    v[0, 322, 0, 7] = math.inf                         # in the open block
    k = k.clamp(-info.max, info.max).where(torch.isfinite(k), k)
    c = kv.new_cache(1, H, D, 6, dtype)
    cache = on_gpu(c)
    context().kv_append(cache, k.cuda(), v.cuda())
    kv.append(c, k, v)
    same_cache(cache, c, "extremes")


def test_append_strides_and_pages_that_are_none():
    say("append strides, bad pages")
    D, H, B, n = 96, 3, 2, 150
    g = torch.Generator().manual_seed(11)
    c = kv.new_cache(B, H, D, 2, HF, pages=12)
    c["table"][0, 1, 0], c["table"][1, 2, 1], c["table"][1, 0, 0] = -1, 12, 2 ** 31 - 1   # the third block of n has no entry at all
    cache = on_gpu(c)
    both = torch.randn(B, H, n, 2, D, generator=g).to(HF)
    k, v = both[:, :, :, 0].transpose(1, 2), both[:, :, :, 1].transpose(1, 2)
    gpu = both.cuda()
    context().kv_append(cache, gpu[:, :, :, 0].transpose(1, 2), gpu[:, :, :, 1].transpose(1, 2))
    kv.append(c, k, v)
    same_cache(cache, c, "strides")
    # lengths outside the table's: below zero counts as zero, above as full; nothing is written past the end
    for length in (-5, 10 ** 6):
        c["lens"].fill_(length)
        cache.lens.fill_(length)
        context().kv_append(cache, gpu[:, :, :, 1].transpose(1, 2), gpu[:, :, :, 0].transpose(1, 2))
        kv.append(c, v, k)
        same_cache(cache, c, "length %d" % length)


# ---- attend


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D,H,g,n,lens,counts", [
    (128, 2, 4, 1, [0, 1, 63, 64, 65, 500], None),
    (64, 1, 1, 1, [129], None),
    (96, 3, 5, 1, [200, 1000], None),
    (128, 1, 16, 1, [300], None),
    (64, 2, 17, 2, [130, 66], None),
    (128, 2, 3, 4, [64, 67, 300, 3], [4, 1, 0, 3]),
    (96, 1, 8, 7, [448, 65], None),
    (64, 2, 2, 70, [70, 200], [70, 33]),
    (128, 1, 4, 130, [130], None),
    (96, 2, 3, 200, [700, 199], [200, 128]),
    (128, 1, 2, 300, [333, 1000], [300, 1]),
    (64, 1, 40, 20, [100], None),
])
def test_attend(dtype, D, H, g, n, lens, counts):
    say("attend", dtype, D, H, g, n, lens, counts)
    c, rand = filled(dtype, D, H, lens, seed=n + D, evicted=[(i + 1) % 2 for i in range(len(lens))], blocks=max(lens) // 64 + 1 + n % 2)
    q = queries(rand, dtype, len(lens), n, H * g, D)
    cnt = None if counts is None else torch.tensor(counts, dtype=torch.int32)
    cache, ctx, gc = on_gpu(c), context(), None if cnt is None else cnt.cuda()
    want = kv.attend(c, q, D ** -0.5, cnt)
    lse = torch.full((len(lens), n, H * g), 7.0, device="cuda")
    out = ctx.kv_attend(cache, q.cuda(), counts=gc, lse=lse)
    check_out(want, out, dtype, "attend", lse)
    mass = torch.full(tuple(c["table"].shape), 7.0, device="cuda")
    out2 = ctx.kv_attend(cache, q.cuda(), counts=gc, mass_out=mass)
    check_out(want, out2, dtype, "attend with weights", mass=mass)
    again = mass.clone()
    ctx.kv_attend(cache, q.cuda(), counts=gc, mass_in=again, mass_out=again)
    torch.testing.assert_close(again, 2 * mass, rtol=1e-6, atol=0)
    lists = torch.arange(c["table"].shape[2], dtype=torch.int32).expand(len(lens), n, H, -1).contiguous()
    lse.fill_(7.0)
    check_out(want, ctx.kv_attend(cache, q.cuda(), counts=gc, lists=lists.cuda(), lse=lse), dtype, "attend, every block listed", lse)


@pytest.mark.parametrize("scale,size", [(1e-3, 1.0), (1.0, 30.0), (20.0, 1.0)])
def test_attend_small_and_large_logits(scale, size):
    say("logits", scale, size)
    for dtype in (BF, HF):
        c, rand = filled(dtype, 64, 1, [333], seed=5)
        q = queries(rand, dtype, 1, 3, 4, 64, size)
        want = kv.attend(c, q, scale)
        lse = torch.empty(1, 3, 4, device="cuda")
        check_out(want, context().kv_attend(on_gpu(c), q.cuda(), scale=scale, lse=lse), dtype, "logits", lse)


def test_attend_many_ranges_join():
    """One long sequence, whose blocks go to many workgroups, beside short and empty ones; the same bits each time."""
    say("ranges")
    for dtype, D, n, g in ((BF, 128, 1, 2), (HF, 64, 2, 5)):
        lens = [20000, 3, 700, 2]
        c, rand = filled(dtype, D, 1, lens, seed=6)
        c["lens"][3] = 0
        q = queries(rand, dtype, 4, n, g, D)
        want = kv.attend(c, q, D ** -0.5)
        cache, ctx = on_gpu(c), context()
        mass, lse = torch.empty(tuple(c["table"].shape), device="cuda"), torch.empty(4, n, g, device="cuda")
        first = ctx.kv_attend(cache, q.cuda(), lse=lse, mass_out=mass)
        check_out(want, first, dtype, "ranges", lse, mass)
        for _ in range(3):
            assert torch.equal(ctx.kv_attend(cache, q.cuda()), first)


def test_attend_strided_queries():
    say("strided queries")
    c, rand = filled(BF, 96, 2, [150, 90], seed=7)
    wide = torch.randn(2, 6, 5, 192, generator=rand).to(BF)          # [B][Hq][n][2 D]
    q = wide[..., 96:].transpose(1, 2)
    want = kv.attend(c, q, 96 ** -0.5)
    gq = wide.cuda()[..., 96:].transpose(1, 2)
    assert not gq.is_contiguous()
    check_out(want, context().kv_attend(on_gpu(c), gq), BF, "strides")
    lists = context().kv_select(on_gpu(c), gq, 2)
    assert torch.equal(lists.cpu(), kv.select(c, q, 2, 0, 0))


def test_attend_pages_that_are_none_and_rows_that_see_nothing():
    say("bad pages, empty rows")
    for dtype in (BF, HF):
        c, rand = filled(dtype, 64, 2, [300, 128, 64], seed=8)
        c["table"][0, 0, 1], c["table"][0, 1, 3], c["table"][2, 0, 0] = -1, c["k"].shape[0], -7
        c["table"][1] = -1                                   # a sequence without a block: its rows see nothing
        q = queries(rand, dtype, 3, 2, 6, 64)
        want = kv.attend(c, q, 0.125)
        cache, ctx = on_gpu(c), context()
        lse, mass = torch.empty(3, 2, 6, device="cuda"), torch.empty(3, 2, 5, device="cuda")
        out = ctx.kv_attend(cache, q.cuda(), lse=lse, mass_out=mass)
        check_out(want, out, dtype, "bad pages", lse, mass)
        assert torch.equal(out[1].cpu(), torch.zeros_like(out[1].cpu())) and (lse[1] == -math.inf).all()
        lists = ctx.kv_select(cache, q.cuda(), 4, sink=1)
        assert torch.equal(lists.cpu(), kv.select(c, q, 4, 1, 0))
        check_out(kv.attend(c, q, 0.125, lists=lists.cpu()), ctx.kv_attend(cache, q.cuda(), lists=lists, lse=lse), dtype, "bad pages listed", lse)
        # lengths outside the table's, more query tokens than the cache has
        c["lens"].copy_(torch.tensor([-3, 1, 2 ** 31 - 1]))
        cache.lens.copy_(c["lens"])
        c["tail_k"].nan_to_num_(0.5)
        c["tail_v"].nan_to_num_(0.5)
        cache.tail_k.nan_to_num_(0.5)
        cache.tail_v.nan_to_num_(0.5)
        check_out(kv.attend(c, q, 0.125), ctx.kv_attend(cache, q.cuda(), lse=lse), dtype, "lengths", lse)


def test_a_token_that_is_not_finite_is_seen_by_its_rows_only():
    say("not finite")
    for dtype in (BF, HF):
        D, H, n = 64, 1, 200
        g = torch.Generator().manual_seed(12)
        k, v, q = (torch.randn(1, n, H, D, generator=g).to(dtype) for _ in range(3))
        for t, what in ((70, math.nan), (198, math.inf)):         # in a full block, in the open one
            kk, vv = k.clone(), v.clone()
            (kk if t == 198 else vv)[0, t, 0, 5] = what
            c = kv.new_cache(1, H, D, 4, dtype)
            cache, ctx = on_gpu(c), context()
            ctx.kv_append(cache, kk.cuda(), vv.cuda())
            kv.append(c, kk, vv)
            cache.lens += n
            c["lens"] += n
            out = ctx.kv_attend(cache, q.cuda())
            assert torch.isnan(out[0, t:].float()).all()
            want = kv.attend(c, q, 0.125)
            for name in want:
                if name != "mass":
                    want[name] = want[name][:, :t]
            check_out(want, out[:, :t], dtype, "rows before")
            # a single late row in a launch of its own
            assert torch.isnan(ctx.kv_attend(cache, q[:, -1:].cuda()).float()).all()


def test_queries_that_are_not_finite_stay_in_their_rows():
    say("queries not finite")
    c, rand = filled(BF, 64, 2, [300], seed=13)
    q = queries(rand, BF, 1, 3, 8, 64)
    want = kv.attend(c, q, 0.125)
    q2 = q.clone()
    q2[0, 1, 2, 7] = math.nan
    out = context().kv_attend(on_gpu(c), q2.cuda())
    assert torch.isnan(out[0, 1, 2].float()).all()
    out[0, 1, 2] = want["out"][0, 1, 2].to(BF).cuda()
    check_out(want, out, BF, "others")


def test_pages_past_32_bits():
    """A pool whose last pages start past 2^32 bytes, and pages whose offset passes 2^31 elements."""
    say("pages past 32 bits")
    D, H, pages = 128, 1, (1 << 32) // (64 * 128) + 3
    ctx = context()
    g = torch.Generator().manual_seed(14)
    n = 64 * 3 + 5
    k, v = (torch.randn(1, n, H, D, generator=g).to(BF) for _ in range(2))
    table = torch.tensor([[[pages - 1, 7, pages - 2, -1]]], dtype=torch.int32)
    small = kv.new_cache(1, H, D, 4, BF, pages=4)
    kv.append(small, k, v)
    small["lens"] += n
    q = queries(g, BF, 1, 2, 4, D)
    e4m3 = torch.float8_e4m3fn
    cache = etf.KvCache(torch.empty(pages, 64, D, dtype=e4m3, device="cuda"), torch.empty(pages, D, 64, dtype=e4m3, device="cuda"), torch.empty(pages, 2, device="cuda"),
                        torch.empty(pages, 2, D, dtype=e4m3, device="cuda"), torch.zeros(1, H, 2, 64, D, dtype=BF, device="cuda"),
                        torch.zeros(1, H, 2, D, 64, dtype=BF, device="cuda"), table.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"),
                        torch.zeros(1, dtype=torch.int32, device="cuda"))
    ctx.kv_append(cache, k.cuda(), v.cuda())
    cache.lens += n
    check_out(kv.attend(small, q, D ** -0.5), ctx.kv_attend(cache, q.cuda()), BF, "far pages")
    assert torch.equal(ctx.kv_select(cache, q.cuda(), 2).cpu(), kv.select(small, q, 2, 0, 0))
    del cache
    torch.cuda.empty_cache()


# ---- select


@pytest.mark.parametrize("dtype,D,H,g,n,lens,counts,w,sink,recent", [
    (BF, 128, 2, 4, 1, [0, 63, 64, 1000, 2000], None, 4, 1, 1),
    (HF, 64, 1, 1, 3, [700, 200], [3, 1], 5, 0, 0),
    (BF, 96, 2, 3, 90, [640, 90], [90, 50], 3, 1, 2),
    (HF, 128, 1, 16, 2, [1500], None, 1, 0, 0),
    (BF, 64, 1, 20, 1, [1280], None, 20, 2, 3),
    (BF, 64, 1, 2, 1, [640], None, 64, 0, 0),
    (BF, 64, 2, 2, 1, [64 * 300 + 3], None, 17, 1, 1),
])
def test_select_and_attend(dtype, D, H, g, n, lens, counts, w, sink, recent):
    say("select", dtype, D, H, g, n, lens, counts, w, sink, recent)
    c, rand = filled(dtype, D, H, lens, seed=20 + w, evicted=[1] * len(lens))
    q = queries(rand, dtype, len(lens), n, H * g, D, 2.0)
    cnt = None if counts is None else torch.tensor(counts, dtype=torch.int32)
    cache, ctx, gc = on_gpu(c), context(), None if cnt is None else cnt.cuda()
    lists = ctx.kv_select(cache, q.cuda(), w, sink=sink, recent=recent, counts=gc)
    want = kv.select(c, q, w, sink, recent, cnt)
    assert torch.equal(lists.cpu(), want)
    lse = torch.empty(len(lens), n, H * g, device="cuda")
    out = ctx.kv_attend(cache, q.cuda(), counts=gc, lists=lists, lse=lse)
    check_out(kv.attend(c, q, D ** -0.5, cnt, want), out, dtype, "listed", lse)


def test_select_ties_go_to_the_lower_block():
    say("ties")
    c, rand = filled(BF, 64, 1, [64 * 700], seed=30)
    for name in ("bounds", "scales"):
        c[name][:] = c[name][int(c["table"][0, 0, 5])]
    q = queries(rand, BF, 1, 2, 2, 64)
    for w, sink, recent in ((3, 0, 0), (300, 0, 1), (5, 2, 2)):
        lists = context().kv_select(on_gpu(c), q.cuda(), w, sink=sink, recent=recent)
        assert torch.equal(lists.cpu(), kv.select(c, q, w, sink, recent))
        assert lists[0, 0, 0].tolist()[: w - recent] == list(range(w - recent))
    q.zero_()
    assert context().kv_select(on_gpu(c), q.cuda(), 4)[0, 0, 0].tolist() == [0, 1, 2, 3]


def test_select_decides_what_float32_cannot():
    """Blocks whose scores differ by less than a float32 sum resolves: a large pair of products cancels and a small one decides."""
    say("near ties")
    c, _ = filled(BF, 64, 1, [64 * 40], seed=31)
    q = torch.zeros(1, 1, 1, 64, dtype=BF)
    q[..., 0], q[..., 1], q[..., 2] = 2.0 ** 14, 2.0 ** 14, 2.0 ** -9
    b = torch.zeros(c["bounds"].shape)
    for j in range(40):
        page = int(c["table"][0, 0, j])
        b[page, :, 0], b[page, :, 1], b[page, :, 2] = 448.0, -448.0, 0.25 * ((j * 17) % 8) + 8
    c["bounds"].copy_(b.to(torch.float8_e4m3fn))
    c["scales"].fill_(1.0)
    for w in (1, 5, 12):
        lists = context().kv_select(on_gpu(c), q.cuda(), w)
        assert torch.equal(lists.cpu(), kv.select(c, q, w, 0, 0))


def bounds_only(D, blocks, whole, distinct, seed, H=1, dtype=BF):
    """A cache whose blocks have bounds and scales (distinct ones, then the same again) and no content."""
    g = torch.Generator().manual_seed(seed)
    table = torch.randint(0, distinct, (1, H, blocks), generator=g) if distinct < whole else torch.randperm(distinct, generator=g)[:blocks].expand(1, H, -1).clone()
    c = kv.new_cache(1, H, D, blocks, dtype, pages=distinct, table=table)
    edges = torch.sort(torch.randn(distinct, 2, D, generator=g) * 100, dim=1)[0].clamp(-448, 448)
    c["bounds"].copy_(edges.to(torch.float8_e4m3fn))
    c["scales"].copy_(torch.exp2(torch.randint(-6, -3, (distinct, 2), generator=g).float()))
    c["lens"][0] = 64 * whole + 7
    return c, g


@pytest.mark.parametrize("blocks,whole,distinct,w", [(300, 256, 300, 9), (1100, 1030, 1100, 40), (1100, 1090, 30, 100), (4200, 4100, 4200, 64), (4200, 4097, 5, 1000),
                                                     (17000, 16500, 17000, 100), (17000, 2100, 17000, 3000), (17000, 16390, 60, 300)])
def test_select_from_long_tables(blocks, whole, distinct, w):
    say("long tables", blocks, whole, distinct, w)
    c, g = bounds_only(64, blocks, whole, distinct, 70 + w)
    c["table"][0, 0, 11], c["table"][0, 0, whole - 3] = -1, distinct
    q = queries(g, BF, 1, 2, 3, 64)
    lists = context().kv_select(on_gpu(c), q.cuda(), w, sink=2, recent=1)
    assert torch.equal(lists.cpu(), kv.select(c, q, w, 2, 1))


@pytest.mark.parametrize("dtype", [BF, HF])
def test_select_scores_that_float32_does_not_hold(dtype):
    """Scores past float32's largest, queries that are not finite, a block among many with a scale far above the others'."""
    say("far scores", dtype)
    c, g = bounds_only(96, 300, 290, 300, 80, dtype=dtype)
    q = queries(g, dtype, 1, 4, 2, 96)
    if dtype == BF:
        c["scales"][:, 0] *= 2.0 ** 100
        q[0, 0] *= 2.0 ** 30
        q[0, 1] *= 2.0 ** 100
    c["scales"][int(c["table"][0, 0, 100]), 0] *= 2.0 ** 14
    q[0, 2, 1] = 0
    want = kv.select(c, q, 12, 1, 1)
    assert torch.equal(context().kv_select(on_gpu(c), q.cuda(), 12, sink=1, recent=1).cpu(), want)
    q[0, 3, 0, 5] = math.nan                    # every score is not a number: all equal, and the others' rows stay
    got = context().kv_select(on_gpu(c), q.cuda(), 12, sink=1, recent=1).cpu()
    assert torch.equal(got[:, :3], want[:, :3]) and got[0, 3, 0].tolist() == list(range(11)) + [289]


def test_lists_that_name_no_block_that_is_seen():
    say("odd lists")
    c, rand = filled(HF, 128, 2, [200, 64], seed=32)
    q = queries(rand, HF, 2, 2, 4, 128)
    lists = torch.tensor([3, -1, 1, 100, 2 ** 31 - 1, 0, -2 ** 31], dtype=torch.int32).expand(2, 2, 2, 7).contiguous()
    lse = torch.empty(2, 2, 4, device="cuda")
    out = context().kv_attend(on_gpu(c), q.cuda(), lists=lists.cuda(), lse=lse)
    check_out(kv.attend(c, q, 128 ** -0.5, lists=lists), out, HF, "odd lists", lse)
    none = torch.full((2, 2, 2, 3), -1, dtype=torch.int32)
    out = context().kv_attend(on_gpu(c), q.cuda(), lists=none.cuda(), lse=lse)
    check_out(kv.attend(c, q, 128 ** -0.5, lists=none), out, HF, "empty lists", lse)


# ---- evict


@pytest.mark.parametrize("blocks,lens,budget,sink,recent", [(8, [500, 64, 0, 130], 4, 1, 1), (1, [64], 1, 0, 0), (40, [2500, 700], 10, 2, 3), (700, [64 * 690 + 1], 300, 4, 8),
                                                            (12, [64 * 12 + 63], 5, 0, 0), (8, [500], 8, 1, 1)])
def test_evict(blocks, lens, budget, sink, recent):
    say("evict", blocks, lens, budget, sink, recent)
    B, H = len(lens), 3
    g = torch.Generator().manual_seed(40 + blocks)
    c = kv.new_cache(B, H, 64, blocks, BF)
    c["lens"].copy_(torch.tensor(lens))
    c["evicted"].copy_(torch.randint(0, 9, (B,), generator=g))
    mass = torch.exp(2 * torch.randn(B, H, blocks, generator=g))
    mass[0, 0] = 1.0                                   # ties
    mass[0, 1, blocks // 2 :] = 0.0
    if blocks > 8:
        mass[0, 2, 3], mass[0, 2, 4], mass[0, 2, 5] = math.nan, math.inf, -1.0
    want = kv.evict(c, mass, budget, sink, recent)
    cache, ctx = on_gpu(c), context()
    to = cache.fork()
    kept, freed = ctx.kv_evict(cache, mass.cuda(), budget, sink=sink, recent=recent, to=to)
    for x, y in zip((to.table, to.lens, to.evicted, kept, freed), want):
        assert torch.equal(torch.nan_to_num(x.cpu(), nan=-9.0), torch.nan_to_num(y, nan=-9.0))
    own = mass.cuda()
    kept, freed = ctx.kv_evict(cache, own, budget, sink=sink, recent=recent)
    for x, y in zip((cache.table, cache.lens, cache.evicted, own, freed), want):
        assert torch.equal(torch.nan_to_num(x.cpu(), nan=-9.0), torch.nan_to_num(y, nan=-9.0))


def test_evict_from_long_tables():
    say("long tables")
    for blocks, n in ((1100, 1050), (5000, 4500), (17000, 16400)):
        g = torch.Generator().manual_seed(blocks)
        c = kv.new_cache(1, 2, 64, blocks, BF, pages=8, table=torch.randint(0, 8, (1, 2, blocks), generator=g))
        c["lens"][0] = 64 * n + 1
        mass = torch.randint(0, 500, (1, 2, blocks), generator=g).float()
        want = kv.evict(c, mass, 700, 3, 20)
        cache, ctx = on_gpu(c), context()
        to = cache.fork()
        kept, freed = ctx.kv_evict(cache, mass.cuda(), 700, sink=3, recent=20, to=to)
        for x, y in zip((to.table, to.lens, to.evicted, kept, freed), want):
            assert torch.equal(x.cpu(), y)
        if blocks <= 16384:
            own = mass.cuda()
            kept, freed = ctx.kv_evict(cache, own, 700, sink=3, recent=20)
            for x, y in zip((cache.table, cache.lens, cache.evicted, own, freed), want):
                assert torch.equal(x.cpu(), y)
        else:
            with pytest.raises(etf.EtfError) as e:
                ctx.kv_evict(cache, mass.cuda(), 700)
            assert e.value.code == -1


def test_a_cache_that_is_cut_goes_on():
    """Tokens come, blocks go by their weight, tokens come again: the device's cache and the oracle's stay the same."""
    say("cut and go on")
    D, H, B, blocks = 64, 2, 2, 8
    g = torch.Generator().manual_seed(50)
    c = kv.new_cache(B, H, D, blocks, BF)
    cache, ctx = on_gpu(c), context()
    mass = torch.zeros(B, H, blocks, device="cuda")
    for step, n in enumerate([300, 1, 40, 64, 7, 100, 1]):
        k, v = (torch.randn(B, n, H, D, generator=g).to(BF) for _ in range(2))
        counts = torch.tensor([n, max(1, n // 2)], dtype=torch.int32)
        ctx.kv_append(cache, k.cuda(), v.cuda(), counts=counts.cuda())
        kv.append(c, k, v, counts)
        cache.lens += counts.cuda()
        c["lens"] += counts
        q = queries(g, BF, B, n, H * 2, D)
        want = kv.attend(c, q, D ** -0.5, counts)
        step_mass = torch.empty_like(mass)
        check_out(want, ctx.kv_attend(cache, q.cuda(), counts=counts.cuda(), mass_out=step_mass), BF, "step %d" % step, mass=step_mass)
        mass += step_mass
        was = mass.cpu()
        _, freed = ctx.kv_evict(cache, mass, 4, sink=1, recent=1)
        table, lens, evicted, kept, gone = kv.evict(c, was, 4, 1, 1)
        assert torch.equal(freed.cpu(), gone) and torch.equal(mass.cpu(), kept)
        # pages that were taken out serve again, at the table's end
        free = [[[int(p) for p in gone[b, h] if p >= 0] + sorted(set(range((b * H + h) * blocks, (b * H + h + 1) * blocks)) - set(table[b, h].tolist()) - set(gone[b, h].tolist()))
                 for h in range(H)] for b in range(B)]
        for b in range(B):
            for h in range(H):
                nb = int(lens[b]) // 64
                table[b, h, nb:] = torch.tensor(free[b][h][: blocks - nb], dtype=torch.int32)
        c["table"], c["lens"], c["evicted"] = table, lens, evicted
        cache.table.copy_(table)
        same_cache(cache, c, "step %d" % step)


# ---- streams and graphs


def test_on_a_stream_of_its_own():
    say("stream")
    c, rand = filled(BF, 128, 2, [1000, 333], seed=60)
    q = queries(rand, BF, 2, 1, 8, 128)
    want, lists = kv.attend(c, q, 128 ** -0.5), kv.select(c, q, 4, 1, 1)
    cache, gq = on_gpu(c), q.cuda()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ctx = etf.Context(device=0, stream=side.cuda_stream)
    for _ in range(5):
        out = ctx.kv_attend(cache, gq)
        got = ctx.kv_select(cache, gq, 4, sink=1, recent=1)
        listed = ctx.kv_attend(cache, gq, lists=got)
        torch.randn(1 << 20, device="cuda").mul_(2)          # work of the program's own stream
        side.synchronize()
        check_out(want, out, BF, "stream")
        assert torch.equal(got.cpu(), lists)
        check_out(kv.attend(c, q, 128 ** -0.5, lists=lists), listed, BF, "stream, listed")


def test_a_step_captured_in_a_graph():
    say("graph")
    D, H, B, g = 128, 2, 3, 4
    c, rand = filled(BF, D, H, [200, 63, 500], blocks=10, seed=61)
    start = on_gpu(c)
    k, v = (torch.randn(B, 1, H, D, generator=rand).to(BF).cuda() for _ in range(2))
    q = queries(rand, BF, B, 1, H * g, D).cuda()
    mass0 = torch.zeros(B, H, 10, device="cuda")

    def step(ctx, cache, mass, out, lists):
        ctx.kv_append(cache, k, v)
        cache.lens += 1
        ctx.kv_attend(cache, q, out=out[0], mass_in=mass, mass_out=mass)
        ctx.kv_select(cache, q, 3, sink=1, recent=1, lists=lists)
        ctx.kv_attend(cache, q, lists=lists, out=out[1])
        ctx.kv_evict(cache, mass, 6, sink=1, recent=2)

    def fresh():
        return etf.KvCache(**{n: getattr(start, n).clone() for n in etf.KvCache.FIELDS}), mass0.clone(), (torch.empty_like(q), torch.empty_like(q)), torch.empty(B, 1, H, 3, dtype=torch.int32, device="cuda")

    eager, ctx = fresh(), context()
    results = []
    for _ in range(4):
        step(ctx, *eager)
        results.append([x.clone() for x in (*eager[2], eager[3], eager[1], eager[0].lens, eager[0].table)])
    torch.cuda.synchronize()
    graphed = fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.set_stream(torch.cuda.current_stream().cuda_stream)
        step(ctx, *graphed)
    ctx.set_stream(torch.cuda.current_stream().cuda_stream)
    spare = fresh()
    for want in results:
        graph.replay()
        step(ctx, *spare)                                    # the program's eager work between the replays
        torch.cuda.synchronize()
        for x, y in zip((*graphed[2], graphed[3], graphed[1], graphed[0].lens, graphed[0].table), want):
            assert torch.equal(x, y)


def test_launches_are_timed_under_a_class_of_their_own():
    say("profile")
    c, rand = filled(BF, 64, 1, [100], seed=62)
    ctx, cache = context(), on_gpu(c)
    ctx.profile_enable(True)
    ctx.kv_attend(cache, queries(rand, BF, 1, 1, 2, 64).cuda())
    ms, count = ctx.profile_read()["kv"]
    assert count >= 1 and ms > 0
