"""Evictions from a table whose pages are counted: the oracle by hand, and what the call refuses or takes before anything reaches a GPU."""
import ctypes
import os
import sys

import pytest

torch = pytest.importorskip("torch")
from oracle import kvcache as kv, pages as pg  # noqa: E402
import paper_1509_05186_amd as etf  # noqa: E402

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_oracle_kvcache import fake_cache  # noqa: E402


def test_eviction_that_keeps_pages_ahead_by_hand():
    c = kv.new_cache(1, 1, 64, 8, torch.bfloat16)
    c["lens"][0], c["evicted"][0] = 5 * 64 + 10, 3
    c["table"][0, 0] = torch.tensor([0, 1, 2, 3, 4, 9, -1, 7])
    mass = torch.tensor([[[1.0, 9.0, 5.0, 5.0, 0.0, 0.5, 7.0, 7.0]]])
    table, lens, evicted, kept, freed = pg.evict(c, mass, 3, 1, 1)
    assert table[0, 0].tolist() == [0, 1, 4, 9, -1, 7, -1, -1] and freed[0, 0].tolist() == [2, 3] + [-1] * 6
    assert kept[0, 0].tolist() == [1.0, 9.0, 0.0, 0.5, 0.0, 0.0, 0.0, 0.0] and lens.tolist() == [3 * 64 + 10] and evicted.tolist() == [5]
    assert torch.equal(pg.evict(c, mass, 5, 1, 1)[0], c["table"]) and (kv.evict(c, mass, 5, 1, 1)[0][0, 0, 5:] == -1).all()


def test_what_is_refused_and_taken():
    ctx = etf.Context(device=None)
    c = fake_cache()

    def evict(mass=4096, budget=4, sink=1, recent=1, table=4096, lens=4096, evicted=4096, out=4096, freed=4096, of=c):
        return ctx._lib.etf_kv_evict_ahead(ctx._h, ctypes.addressof(of), mass, budget, sink, recent, table, lens, evicted, out, freed)

    assert evict() == -5
    for bad in (dict(mass=None), dict(budget=0), dict(sink=-1), dict(recent=-2), dict(sink=3, recent=2), dict(table=None), dict(lens=None), dict(evicted=None),
                dict(out=None), dict(freed=None), dict(of=fake_cache(head_dim=80))):
        assert evict(**bad) == -1, bad
    wide = fake_cache(max_blocks=16385)
    assert evict(of=wide) == -1 and evict(of=wide, table=8192, out=8192) == -5 and evict(of=fake_cache(max_blocks=16384)) == -5
    assert ctx._lib.etf_kv_evict_ahead(None, ctypes.addressof(c), 4096, 4, 1, 1, 4096, 4096, 4096, 4096, 4096) == -1
    host = etf.KvCache(**kv.new_cache(2, 3, 64, 4, torch.bfloat16))
    with pytest.raises(etf.EtfError) as e:
        ctx.kv_evict(host, torch.zeros(2, 3, 4), 2, ahead=True)
    assert e.value.code == -5
    with pytest.raises(ValueError, match="mass"):
        ctx.kv_evict(host, torch.zeros(2, 3, 3), 2, ahead=True)
