"""Arguments that the cache calls refuse or take, before anything reaches a GPU (no GPU: what is taken ends with its absence, code -5)."""
import ctypes
import os
import sys

import pytest

torch = pytest.importorskip("torch")
from oracle import kvcache as kv  # noqa: E402
import paper_1509_05186_amd as etf  # noqa: E402

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_oracle_kvcache import fake_cache  # noqa: E402


@pytest.fixture(scope="module")
def made():
    ctx, c = etf.Context(device=None), etf.KvCache(**kv.new_cache(2, 3, 64, 4, torch.bfloat16))
    ws = torch.empty(1 << 16, dtype=torch.uint8)
    q = torch.zeros(2, 1, 6, 64, dtype=torch.bfloat16)
    return ctx, c, q, dict(out=torch.empty_like(q), ws=ws)


def taken(call, *args, **kw):
    with pytest.raises(etf.EtfError) as e:
        call(*args, **kw)
    assert e.value.code == -5


def test_lists_without_an_entry_are_not_all_tokens(made):
    ctx, c, q, room = made
    taken(ctx.kv_attend, c, q, lists=torch.zeros(2, 1, 3, 1, dtype=torch.int32), **room)
    with pytest.raises(ValueError, match="lists"):
        ctx.kv_attend(c, q, lists=torch.zeros(2, 1, 3, 0, dtype=torch.int32), **room)


def test_no_gradient_is_lost_in_silence(made):
    ctx, c, q, room = made
    grad = q.clone().requires_grad_()
    new = torch.zeros(2, 1, 3, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="gradient"):
        ctx.kv_attend(c, grad, **room)
    for k, v in ((new.clone().requires_grad_(), new), (new, new.clone().requires_grad_())):
        with pytest.raises(ValueError, match="gradient"):
            ctx.kv_append(c, k, v)
        with torch.no_grad():
            taken(ctx.kv_append, c, k, v)
        taken(ctx.kv_append, c, k.detach(), v.detach())
    with torch.no_grad():
        taken(ctx.kv_attend, c, grad, **room)
    taken(ctx.kv_attend, c, grad.detach(), **room)
    taken(ctx.kv_select, c, grad, 2, ws=room["ws"], lists=torch.empty(2, 1, 3, 2, dtype=torch.int32))     # block numbers have no gradient


def test_strides_that_no_row_uses_are_not_asked_about(made):
    ctx, c, q, room = made
    wide = torch.zeros(2, 4, 6, 68, dtype=torch.bfloat16)          # rows of 68 elements: no stride of 8
    with pytest.raises(etf.EtfError) as e:
        ctx.kv_attend(c, wide[:, :1, :, :64], **room)
    assert e.value.code == -1
    one = etf.KvCache(**kv.new_cache(1, 1, 64, 4, torch.bfloat16))
    lone = torch.zeros(4 * 132, dtype=torch.bfloat16).as_strided((1, 1, 2, 64), (131, 68, 72, 1))     # one sequence, one token
    assert not lone.is_contiguous()
    out = torch.empty(1, 1, 2, 64, dtype=torch.bfloat16)
    taken(ctx.kv_attend, one, lone, out=out, ws=room["ws"])
    taken(ctx.kv_append, one, lone[:, :, :1].expand(1, 3, 1, 64), torch.zeros(600, dtype=torch.bfloat16).as_strided((1, 3, 1, 64), (1, 136, 3, 1)))
    taken(ctx.kv_select, one, lone, 2, ws=room["ws"], lists=torch.empty(1, 1, 1, 2, dtype=torch.int32))


def test_launches_of_2_to_the_32_threads_are_refused_before_the_first():
    ctx = etf.Context(device=None)
    lib, h, far = ctx._lib, ctx._h, 1 << 60

    def append(n, **over):
        c = fake_cache(**over)
        return lib.etf_kv_append(h, ctypes.addressof(c), 4096, None, 4096, None, n, None)

    def attend(n, group, lists=None, w=0, mass=None, **over):
        c = fake_cache(**over)
        return lib.etf_kv_attend(h, ctypes.addressof(c), 4096, None, n, c.heads * group, 1.0, None, lists, w, 4096, None, None, mass, 4096, far)

    def select(n, **over):
        c = fake_cache(**over)
        return lib.etf_kv_select(h, ctypes.addressof(c), 4096, None, n, c.heads, None, 2, 0, 0, 4096, 4096, far)

    def evict(**over):
        c = fake_cache(**over)
        return lib.etf_kv_evict(h, ctypes.addressof(c), 4096, 4, 1, 1, 4096, 4096, 4096, 4096, 4096)

    # (the last size that is taken, the first that is not), threads of a launch below and at 2^32
    for call, few, many in (
            (append, dict(n=64 * 63, batch=1 << 12, heads=1 << 6), dict(n=64 * 64, batch=1 << 12, heads=1 << 6)),
            (attend, dict(n=1, group=1, batch=1 << 14, heads=1 << 9, max_blocks=32), dict(n=1, group=1, batch=1 << 14, heads=1 << 9, max_blocks=33)),      # joined: two workgroups to a tile
            (attend, dict(n=256, group=1, mass=4096, batch=1 << 6, heads=1 << 3, max_blocks=(1 << 15) - 1), dict(n=256, group=1, mass=4096, batch=1 << 6, heads=1 << 3, max_blocks=1 << 15)),
            (attend, dict(n=1 << 10, group=1, lists=4096, w=2, batch=1 << 10, heads=63), dict(n=1 << 10, group=1, lists=4096, w=2, batch=1 << 10, heads=64)),
            (select, dict(n=1 << 10, batch=1 << 10, heads=63), dict(n=1 << 10, batch=1 << 10, heads=64)),
            (select, dict(n=1 << 10, batch=1 << 7, heads=31, max_blocks=4097), dict(n=1 << 10, batch=1 << 7, heads=32, max_blocks=4097)),
            (evict, dict(batch=1 << 13, heads=(1 << 13) - 1, max_blocks=8), dict(batch=1 << 13, heads=1 << 13, max_blocks=8))):
        assert call(**few) == -5, (call, few)
        assert call(**many) == -1, (call, many)
