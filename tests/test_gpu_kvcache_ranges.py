"""The split of an attention call into ranges, choices among few and many keys, eviction in place and apart, and the example, on the GPU
against the oracle in float64; bounds as in test_gpu_kvcache.py."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import kvcache as kv  # noqa: E402
import paper_1509_05186_amd as etf  # noqa: E402

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_gpu_kvcache import BF, HF, check_out, context, filled, on_gpu, queries, say  # noqa: E402


# counts leave whole tiles of 16 and of 128 rows to padding, of some sequences all; few and many units, rounds of workgroups
@pytest.mark.parametrize("dtype,D,H,g,n,lens,counts", [
    (BF, 128, 1, 4, 300, [2000, 400, 300], [300, 1, 0]),
    (HF, 96, 2, 5, 130, [1500, 131, 700, 64], [0, 130, 27, 64]),
    (BF, 64, 1, 1, 64, [900, 5000], [64, 16]),
    (BF, 128, 2, 8, 8, [3000, 100, 0, 700], [1, 8, 8, 0]),
    (HF, 64, 1, 16, 4, [6000], [3]),
    (BF, 96, 3, 3, 200, [64, 1], [1, 1]),
])
@pytest.mark.parametrize("mass", [False, True])
def test_ranges_and_tiles_of_padding(dtype, D, H, g, n, lens, counts, mass):
    say("ranges", dtype, D, H, g, n, lens, counts, mass)
    c, rand = filled(dtype, D, H, lens, seed=len(lens) * 7 + n)
    q = queries(rand, dtype, len(lens), n, H * g, D)
    cnt = torch.tensor(counts, dtype=torch.int32)
    want = kv.attend(c, q, D ** -0.5, counts=cnt)
    cache = on_gpu(c)
    lse = torch.full(q.shape[:3], 7.0, device="cuda")
    m = torch.full(cache.table.shape, 3.0, device="cuda") if mass else None
    out = context().kv_attend(cache, q.cuda(), counts=cnt.cuda(), lse=lse, out=torch.full_like(q, 5.0, device="cuda"), mass_out=m)
    check_out(want, out, dtype, "ranges", lse, m)
    for b, x in enumerate(counts):
        assert torch.all(out[b, x:] == 0) and torch.all(lse[b, x:] == -math.inf)


# more sequences than a wave has lanes, very short ones beside a long one
@pytest.mark.parametrize("n,g", [(1, 4), (20, 4)])
def test_ranges_of_many_sequences(n, g):
    say("many sequences", n, g)
    D, H = 64, 1
    lens = [1700 if b in (3, 68) else (b * 37) % 200 + n for b in range(70)]
    c, rand = filled(BF, D, H, lens, seed=70)
    q = queries(rand, BF, 70, n, H * g, D)
    lse = torch.empty(q.shape[:3], device="cuda")
    out = context().kv_attend(on_gpu(c), q.cuda(), lse=lse)
    check_out(kv.attend(c, q, D ** -0.5), out, BF, "many sequences", lse)


def evict_in_place_and_apart(c, mass, budget, sink, recent):
    """What kv_evict writes into a fork, and into the cache itself; both have to be the same."""
    apart, place = on_gpu(c), on_gpu(c)
    to, ctx, held = apart.fork(), context(), mass.cuda()
    kept, freed = ctx.kv_evict(apart, held, budget, sink=sink, recent=recent, to=to)
    again, freed2 = ctx.kv_evict(place, held.clone(), budget, sink=sink, recent=recent)
    for x, y in ((to.table, place.table), (to.lens, place.lens), (to.evicted, place.evicted), (kept, again), (freed, freed2)):
        assert torch.equal(x, y)
    assert torch.equal(apart.table.cpu(), c["table"]) and torch.equal(apart.lens.cpu(), c["lens"])
    return to, kept, freed


@pytest.mark.parametrize("blocks,full,budget", [(256, 255, 100), (257, 250, 249), (1024, 1000, 500), (1025, 1024, 64), (5000, 4500, 4000)])
@pytest.mark.parametrize("distinct", [3, 70, 100_000])
def test_evict_by_few_and_many_weights(blocks, full, budget, distinct):
    """Tables on both sides of every kernel's limit; many equal weights, fewer than a wave's lanes between two counts, none equal."""
    say("evict", blocks, full, budget, distinct)
    g = torch.Generator().manual_seed(blocks + distinct)
    table = torch.randperm(blocks * 2, generator=g).view(1, 2, blocks)
    c = kv.new_cache(1, 2, 64, blocks, BF, table=table)
    c["lens"][0] = full * 64 + 9
    c["evicted"][0] = 5
    mass = torch.randint(0, distinct, (1, 2, blocks), generator=g).float() / 8
    to, kept, freed = evict_in_place_and_apart(c, mass, budget, 2, 3)
    for h in range(2):
        rank = sorted(range(2, full - 3), key=lambda j: (-float(mass[0, h, j]), j))[: budget - 5]
        stay = sorted([0, 1, *rank, full - 3, full - 2, full - 1])
        gone = sorted(set(range(full)) - set(stay))
        assert to.table[0, h].tolist() == table[0, h][stay].tolist() + [-1] * (blocks - budget)
        assert freed[0, h].tolist() == table[0, h][gone].tolist() + [-1] * (blocks - len(gone))
        assert kept[0, h].tolist() == mass[0, h][stay].tolist() + ([float(mass[0, h, full])] if full < blocks else []) + [0.0] * (blocks - budget - (full < blocks))
    assert to.lens.tolist() == [budget * 64 + 9] and to.evicted.tolist() == [5 + full - budget]


def test_the_example():
    """The cache stays within its budget; its last attention is off by the roundings of bf16 only: those of the weights and of the output."""
    say("example")
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import bounded_cache
    cache, off = bounded_cache.main(["--batch", "3", "--heads", "2", "--prompt", "1500", "--piece", "300", "--tokens", "150", "--budget", "8", "--w", "4"])
    lens, evicted = cache.cache.lens.tolist(), cache.cache.evicted.tolist()
    assert all(8 * 64 <= x < 8 * 64 + 128 for x in lens) and all(x + 64 * e == 1650 for x, e in zip(lens, evicted))
    # no page is lost or stands twice
    assert sorted(cache.cache.table.flatten().tolist()) == list(range(cache.cache.pages))
    most = float(cache.cache.tail_v.abs().max().clamp_min(448 * cache.cache.scales[:, 1].max()))
    assert off <= 2 * 2.0 ** -8 * most + 2.0 ** -12 * most
