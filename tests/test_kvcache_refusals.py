"""Arguments that the cache calls refuse or take, before anything reaches a GPU (no GPU: what is taken ends with its absence, code -5)."""
import pytest

torch = pytest.importorskip("torch")
from oracle import kvcache as kv  # noqa: E402
import paper_1509_05186_amd as etf  # noqa: E402


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
