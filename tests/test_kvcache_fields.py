"""KvCache's fields and the arrays that the kernels are given stay the same ones (no GPU)."""
import pytest

torch = pytest.importorskip("torch")
from oracle import kvcache as kv  # noqa: E402
import paper_1509_05186_amd as etf  # noqa: E402


def cache():
    return etf.KvCache(**kv.new_cache(2, 3, 64, 4, torch.bfloat16))


def same_arrays(c):
    for name in etf.KvCache.FIELDS:
        assert getattr(c._c, name) == getattr(c, name).data_ptr(), name


def test_a_fork_of_a_cache_that_was_advanced_has_its_own_lengths():
    c = cache()
    c.lens += 100
    c.table += 1
    c.evicted += 2
    to = c.fork()
    same_arrays(c)
    same_arrays(to)
    for name in etf.KvCache.FIELDS:
        assert (getattr(to, name) is getattr(c, name)) == (name not in ("table", "lens", "evicted")), name
    to.lens.zero_()
    to.lens += 7
    assert to.lens.tolist() == [7, 7] and c.lens.tolist() == [100, 100] and c.evicted.tolist() == [2, 2]
    again = to.fork()
    same_arrays(again)
    assert again.lens is not to.lens and again.k is c.k


def test_a_field_that_is_assigned_is_what_the_kernels_are_given():
    c = cache()
    to = c.fork()
    c.lens = c.lens + 5
    c.table = torch.full_like(c.table, 3)
    same_arrays(c)
    same_arrays(to)
    assert c.lens.tolist() == [5, 5] and (c.table == 3).all() and to.lens is not c.lens


def test_assignments_that_do_not_fit_are_refused_and_change_nothing():
    c = cache()
    was = {name: getattr(c, name) for name in etf.KvCache.FIELDS}
    for name, bad in (("lens", c.lens.long()), ("lens", c.lens[:1]), ("lens", 3), ("lens", None), ("table", c.table.transpose(1, 2)),
                      ("table", torch.zeros(2, 3, 5, dtype=torch.int32)), ("k", c.k.float()), ("tail_k", c.tail_k.half()),
                      ("evicted", torch.zeros(4, dtype=torch.int32)[::2])):
        with pytest.raises(ValueError):
            setattr(c, name, bad)
        assert all(getattr(c, x) is was[x] for x in was)
        same_arrays(c)
    with pytest.raises(AttributeError):
        del c.lens
