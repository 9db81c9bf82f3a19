"""Appends, packed and padded, at both parities of the open block's buffer and with tokens that are not finite in every place that the kernel takes them
from: the open block, the blocks that are completed, and what is left over, below eight tokens and above.  Numbers equal the oracle's; what is not a
number is so in both."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import kvcache as kv  # noqa: E402
import paper_1509_05186_amd as etf  # noqa: E402

BF, HF = torch.bfloat16, torch.float16

# open tokens and new ones: a few into the open block (one wave), more of them, blocks completed with nothing, few and many left over, two and three
# blocks at once (the open block's buffer is then the same, or the other one)
CASES = [(0, 1), (5, 4), (60, 3), (5, 7), (3, 40), (63, 1), (60, 4), (60, 9), (60, 12), (10, 100), (0, 64), (1, 130), (33, 160), (64 + 40, 24), (128 + 7, 57 + 64 + 20), (64, 0), (70, 5)]


def say(*a):
    print(*a, flush=True)


def equal(x, y):
    x, y = x.cpu().float(), y.float()
    return torch.equal(x.isnan(), y.isnan()) and torch.equal(torch.nan_to_num(x, nan=0.0), torch.nan_to_num(y, nan=0.0))


@pytest.mark.parametrize("dtype,D,H", [(BF, 128, 2), (HF, 96, 3), (BF, 64, 1), (HF, 64, 2)])
@pytest.mark.parametrize("evicted", [0, 1, 2, 7])
@pytest.mark.parametrize("bad", [False, True])
def test_every_place_and_both_buffers(dtype, D, H, evicted, bad):
    say("append", dtype, D, H, "evicted", evicted, "bad", bad)
    check(CASES, dtype, D, H, evicted, bad)


@pytest.mark.parametrize("dtype,D,H", [(BF, 128, 1), (HF, 96, 2), (BF, 64, 1)])
@pytest.mark.parametrize("sealed", [0, 1, 2])
def test_both_sides_of_a_few_tokens(dtype, D, H, sealed):
    """What is left over is written token by token up to 16, 20 and 32 of them (128, 96 and 64 dimensions), and turned first from there on; at every
    place in its block that pieces of eight tokens begin or end."""
    say("a few", dtype, D, H, sealed)
    few = {128: 16, 96: 20, 64: 32}[D]
    over = [few - 1, few, few + 1, few + 2, few + 5, few + 9]
    cases = [(61, 3 + 64 * (sealed - 1) + n) for n in over + [63]] if sealed else [(begin, n) for n in over for begin in (0, 1, 2, 3, 5, 6, 7, 8, 17, 22)]
    for bad in (False, True):
        check(cases, dtype, D, H, 1, bad)


def check(cases, dtype, D, H, evicted, bad):
    lens, counts = (list(x) for x in zip(*cases))
    B = len(cases)
    g = torch.Generator().manual_seed(D + evicted)
    made = lambda n: [torch.randn(B, n, H, D, generator=g).to(dtype) for _ in range(2)]  # noqa: E731

    def spoil(k, v, tokens):
        """Some of each sequence's tokens, the first and the last among them in turn, get a key or value that is not finite."""
        for b, n in enumerate(tokens):
            for i in {0, n // 2, n - 1} if b % 2 else {n - 1}:
                if n:
                    x = (k, v)[(b + i) % 2]
                    x[b, i, b % H, (7 * b + i) % D] = (math.nan, math.inf, -math.inf)[(b + i) % 3]

    c = kv.new_cache(B, H, D, 6, dtype, table=torch.randperm(B * H * 6, generator=g).view(B, H, 6))
    c["evicted"].fill_(evicted)
    c["evicted"][::3] += 1
    before = made(max(lens))
    if bad:
        spoil(*before, lens)
    kv.append(c, *before, torch.tensor(lens))
    c["lens"].copy_(torch.tensor(lens))
    k, v = made(max(counts))
    if bad:
        spoil(k, v, counts)
    start = {name: c[name].clone() for name in etf.KvCache.FIELDS}
    on_gpu = lambda: etf.KvCache(**{name: start[name].cuda() for name in etf.KvCache.FIELDS})  # noqa: E731
    ctx = etf.Context(device=0, stream=torch.cuda.current_stream().cuda_stream)
    padded, packed = on_gpu(), on_gpu()
    ctx.kv_append(padded, k.cuda(), v.cuda(), counts=torch.tensor(counts, dtype=torch.int32, device="cuda"))
    lie = lambda x: torch.cat([x[b, :n] for b, n in enumerate(counts)]).cuda()  # noqa: E731
    starts = torch.tensor([0] + counts, device="cuda").cumsum(0).to(torch.int32)
    ctx.kv_append_packed(packed, lie(k), lie(v), starts)
    kv.append(c, k, v, torch.tensor(counts))
    torch.cuda.synchronize()
    for cache in (padded, packed):
        for name in etf.KvCache.FIELDS:
            assert equal(getattr(cache, name), c[name]), name


@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 96)])
def test_attention_after_appends_to_either_buffer(dtype, D):
    """The open block is read from where an append has put it."""
    say("append and attend", dtype, D)
    B, H, g = 4, 2, 2
    gen = torch.Generator().manual_seed(D)
    ctx = etf.Context(device=0, stream=torch.cuda.current_stream().cuda_stream)
    caches = []
    for evicted in (0, 1):
        cache = etf.KvCache.alloc(B, H, D, 640, dtype=dtype)
        cache.evicted.fill_(evicted)
        caches.append(cache)
    for n in (40, 3, 30, 64, 100, 1, 130):
        k, v = (torch.randn(B, n, H, D, generator=gen).to(dtype).cuda() for _ in range(2))
        for cache in caches:
            ctx.kv_append(cache, k, v)
            cache.lens += n
        q = torch.randn(B, 1, H * g, D, generator=gen).to(dtype).cuda()
        assert torch.equal(*(ctx.kv_attend(cache, q) for cache in caches)), n
