"""Arguments that packed prompts' attention and the calls on a cache's pages refuse or take, before anything reaches a GPU (no GPU: what is taken ends
with its absence, code -5)."""
import ctypes
import os
import sys

import pytest

torch = pytest.importorskip("torch")
from oracle import kvcache as kv  # noqa: E402
import paper_1509_05186_amd as etf  # noqa: E402

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_oracle_kvcache import fake_cache  # noqa: E402

BF, HF, I32 = torch.bfloat16, torch.float16, torch.int32


@pytest.fixture(scope="module")
def ctx():
    return etf.Context(device=None)


def taken(call, *args, **kw):
    with pytest.raises(etf.EtfError) as e:
        call(*args, **kw)
    assert e.value.code == -5


def refused(call, *args, match=None, **kw):
    with pytest.raises((ValueError, etf.EtfError), match=match) as e:
        call(*args, **kw)
    assert not isinstance(e.value, etf.EtfError) or e.value.code in (-1, -3), e.value


def prompt(T=10, Hq=6, H=3, D=64, dtype=BF):
    return [torch.zeros(T, x, D, dtype=dtype) for x in (Hq, H, H)] + [torch.tensor([0, 4, T], dtype=I32)]


# ---- attention of prompts


def test_prompts_are_taken(ctx):
    for dtype in (BF, HF):
        for D in (64, 96, 128):
            taken(ctx.prompt_attend, *prompt(D=D, dtype=dtype))
    q, k, v, st = prompt()
    taken(ctx.prompt_attend, q, k, v, st, scale=2.0, out=torch.empty_like(q), lse=torch.empty(10, 6), ws=torch.empty(1024, dtype=torch.uint8))
    fused = torch.zeros(10, 12, 64, dtype=BF)
    taken(ctx.prompt_attend, fused[:, :6], fused[:, 6:9], fused[:, 9:], st)
    taken(ctx.prompt_attend, q, k[:, :1].expand(10, 3, 64), v, st)
    one = torch.zeros(4 * 100, dtype=BF)
    taken(ctx.prompt_attend, one.as_strided((1, 1, 64), (7, 3, 1)), one.as_strided((1, 1, 64), (5, 5, 1)), one[:64].view(1, 1, 64), torch.tensor([0, 1], dtype=I32))     # strides that no row uses


def test_prompts_of_other_shapes_and_types_are_refused(ctx):
    q, k, v, st = prompt()
    for bad in (q.float(), q[:, :, :63], q[0], q[:, :5], q[:9], q.half()):
        refused(ctx.prompt_attend, bad, k, v, st)
    for bad in (k[:, :2], k[:9], k.half(), torch.zeros(10, 3, 96, dtype=BF), k[:, :, :32], k.transpose(1, 2)):
        refused(ctx.prompt_attend, q, bad, v, st)
        refused(ctx.prompt_attend, q, k, bad, st)
    for bad in (st[:1], st.long(), st[None], torch.zeros(6, dtype=I32)[::2]):
        refused(ctx.prompt_attend, q, k, v, bad, match="starts")
    for bad in (torch.empty(10, 6, 64), torch.empty(10, 6, 65, dtype=BF), torch.empty(10, 12, 64, dtype=BF)[:, ::2]):
        refused(ctx.prompt_attend, q, k, v, st, out=bad, match="out")
    for bad in (torch.empty(10, 3), torch.empty(10, 6, dtype=torch.float64)):
        refused(ctx.prompt_attend, q, k, v, st, lse=bad, match="lse")
    for D in (32, 80, 256):
        refused(ctx.prompt_attend, *prompt(D=D), match="head_dim")
    refused(ctx.prompt_attend, *prompt(Hq=5), match="multiple")
    refused(ctx.prompt_attend, *prompt(T=10)[:3], torch.zeros(2, dtype=I32), scale=0.0, match="scale")
    refused(ctx.prompt_attend, q, k, v, st, scale=float("inf"), match="scale")
    refused(ctx.prompt_attend, q[:0], k[:0], v[:0], st, match="positive")
    wide = torch.zeros(10, 6, 68, dtype=BF)
    refused(ctx.prompt_attend, wide[:, :, :64], k, v, st, match="stride")
    refused(ctx.prompt_attend, torch.zeros(10 * 6 * 64 + 4, dtype=BF)[4:].view(10, 6, 64), k, v, st, match="aligned")
    refused(ctx.prompt_attend, q, torch.zeros(1, dtype=BF).as_strided((10, 3, 64), (0, 0, 0)), v, st, match="contiguous")


def test_prompts_whose_gradient_would_be_lost_are_refused(ctx):
    for i in range(3):
        x = prompt()
        x[i].requires_grad_()
        with pytest.raises(ValueError, match="gradient"):
            ctx.prompt_attend(*x)
        with torch.no_grad():
            taken(ctx.prompt_attend, *x)
    c = etf.KvCache(**kv.new_cache(2, 3, 64, 4, BF))
    with pytest.raises(ValueError, match="gradient"):
        ctx.kv_append_packed(c, prompt()[1].requires_grad_(), prompt()[2], prompt()[3])


def test_prompts_of_the_largest_sizes(ctx):
    lib, h, size = ctx._lib, ctx._h, 1 << 60

    def call(dtype=0, D=64, qs=None, ks=None, tokens=100, hq=2, heads=1, batch=2, scale=1.0, q=4096, starts=4096, out=4096, ws=4096, nws=size):
        s = lambda x: None if x is None else (ctypes.c_int64 * 2)(*x)  # noqa: E731
        return lib.etf_prompt_attend(h, dtype, D, q, s(qs), 4096, s(ks), 4096, None, tokens, hq, heads, starts, batch, scale, out, None, ws, nws)

    assert call() == -5 and call(dtype=1) == -5 and call(dtype=2) == -1 and call(q=None) == -1 and call(q=4100) == -1 and call(starts=None) == -1 and call(out=4104) == -1
    assert call(qs=(128, 64)) == -5 and call(qs=(124, 64)) == -1 and call(qs=(128, -8)) == -1 and call(ks=(1 << 23, 1 << 40)) == -5 and call(ks=((1 << 23) + 8, 64)) == -1
    # a workgroup to 128 rows and one to each sequence, fewer than 2^24 of them
    assert call(tokens=(1 << 30) - 256) == -5 and call(tokens=1 << 30) == -1 and call(batch=1 << 24) == -1 and call(batch=(1 << 23) - 1, heads=2) == -5 and call(batch=1 << 23, heads=2) == -1
    assert call(tokens=4000, hq=1) == -5 and call(tokens=4000, hq=1, ws=None) == -1 and call(tokens=4000, hq=1, ws=4100) == -1 and call(tokens=4000, hq=1, nws=1024) == -3
    assert call(ws=None, nws=0) == -5      # no ranges: no workspace
    assert lib.etf_prompt_attend_workspace_bytes(h, 64, 100, 2, 1, 2) == 0 and lib.etf_prompt_attend_workspace_bytes(h, 64, 4000, 1, 1, 1) > 0
    assert lib.etf_prompt_attend_workspace_bytes(h, 63, 100, 2, 1, 2) == -1 and lib.etf_prompt_attend_workspace_bytes(None, 64, 100, 2, 1, 2) == -1
    assert lib.etf_prompt_attend(None, 0, 64, 4096, None, 4096, None, 4096, None, 1, 1, 1, 4096, 1, 1.0, 4096, None, None, 0) == -1


# ---- appends of packed tokens, pages


def test_pages_are_taken_and_refused(ctx):
    c = etf.KvCache(**kv.new_cache(2, 3, 64, 4, BF))
    refs, ws = torch.zeros(c.pages, dtype=I32), torch.empty(1 << 16, dtype=torch.uint8)
    k, st = torch.zeros(9, 3, 64, dtype=BF), torch.tensor([0, 4, 9], dtype=I32)
    two, table = torch.zeros(2, dtype=I32), torch.empty_like(c.table)
    taken(ctx.kv_append_packed, c, k, k, st)
    taken(ctx.kv_append_packed, c, k[:, :1].expand(9, 3, 64), torch.zeros(9, 6, 64, dtype=BF)[:, 3:], st)
    for bad in (k[:8], k[:, :2], k.half(), k[0], k[None]):
        refused(ctx.kv_append_packed, c, k, bad, st)
    refused(ctx.kv_append_packed, c, k.half(), k.half(), st)
    refused(ctx.kv_append_packed, c, k[:0], k[:0], st, match="tokens")
    for bad in (st[:2], st.long()):
        refused(ctx.kv_append_packed, c, k, k, bad, match="starts")
    taken(ctx.kv_take, c, refs)
    taken(ctx.kv_take, c, refs, 1 << 24, counts=two, table_out=table, refs_out=torch.empty_like(refs), missing=torch.zeros(1, dtype=I32), ws=ws)
    refused(ctx.kv_take, c, refs, 0, match="n")
    refused(ctx.kv_take, c, refs, (1 << 24) + 1, match="n")
    for kw in (dict(counts=two[:1]), dict(counts=two.long()), dict(table_out=table[:1]), dict(refs_out=refs[:-1]), dict(missing=two), dict(ws=ws[:300])):
        refused(ctx.kv_take, c, refs, **kw)
    for bad in (refs[:-1], refs.long(), torch.zeros(c.pages + 1, dtype=I32)):
        refused(ctx.kv_take, c, bad, match="refs")
        refused(ctx.kv_fork, c, bad, two, match="refs")
        refused(ctx.kv_compact, c, bad, match="refs")
    taken(ctx.kv_fork, c, refs, two)
    taken(ctx.kv_fork, c, refs, two, keep=two)
    for bad in (two[:1], two.long(), table):
        refused(ctx.kv_fork, c, refs, bad, match="source")
        refused(ctx.kv_fork, c, refs, two, keep=bad, match="keep")
    refused(ctx.kv_fork, c, refs, two, ws=ws[:1000])
    taken(ctx.kv_compact, c, refs)
    taken(ctx.kv_compact, c, refs, table_out=table, refs_out=torch.empty_like(refs), used=torch.zeros(1, dtype=I32), ws=ws)
    for kw in (dict(table_out=table.long()), dict(refs_out=refs[:-1]), dict(used=two), dict(ws=ws[:256])):
        refused(ctx.kv_compact, c, refs, **kw)
    taken(ctx.kv_free, refs, table)
    taken(ctx.kv_free, refs, two[:0])
    for bad in (table.long(), c.table[:, ::2]):
        refused(ctx.kv_free, refs, bad, match="pages")
    for bad in (refs.long(), refs[::2], table, refs[:0]):
        refused(ctx.kv_free, bad, two)


def test_pages_of_the_largest_sizes(ctx):
    lib, h, far = ctx._lib, ctx._h, 1 << 60

    def of(call, *args, **over):
        c = fake_cache(**over)
        return getattr(lib, call)(h, ctypes.addressof(c), *args)

    take = lambda n=1, refs=4096, **o: of("etf_kv_take", refs, n, None, 4096, 4096, 4096, 4096, far, **o)  # noqa: E731
    fork = lambda **o: of("etf_kv_fork", 4096, 4096, None, 4096, far, **o)  # noqa: E731
    compact = lambda **o: of("etf_kv_compact", 4096, 4096, 4096, 4096, 4096, far, **o)  # noqa: E731
    append = lambda tokens, **o: of("etf_kv_append_packed", 4096, None, 4096, None, tokens, 4096, **o)  # noqa: E731
    assert take() == -5 and fork() == -5 and compact() == -5 and append(10) == -5
    most = dict(batch=1 << 12, heads=1 << 8, max_blocks=(1 << 11) - 1, pages=(1 << 31) - 1)
    assert take(1 << 24, **most) == -5 and compact(**most) == -5
    assert fork(batch=1 << 12, heads=1365, max_blocks=8) == -5 and fork(batch=1 << 12, heads=1366, max_blocks=8) == -1      # three workgroups to a row
    assert append((1 << 30) - 200, batch=1, heads=1) == -5 and append(1 << 30, batch=1, heads=1) == -1 and append(0) == -1
    assert append(64 * 1023, batch=1 << 12, heads=3277) == -5 and append(64 * 1024, batch=1 << 12, heads=3277) == -1
    for over in (dict(head_dim=80), dict(dtype=2), dict(batch=0), dict(pages=0), dict(max_blocks=1 << 30), dict(table=None), dict(k=4100)):
        assert take(**over) == -1 and fork(**over) == -1 and compact(**over) == -1 and append(10, **over) == -1, over
    assert take(refs=None) == -1
    assert lib.etf_kv_free(h, 4096, 5, 4096, 1 << 20) == -5 and lib.etf_kv_free(h, 4096, 0, 4096, 1) == -1 and lib.etf_kv_free(h, None, 5, 4096, 1) == -1
    assert lib.etf_kv_free(h, 4096, 5, None, 1) == -1 and lib.etf_kv_free(h, 4096, 5, 4096, -1) == -1 and lib.etf_kv_free(h, 4096, 5, 4096, 1 << 40) == -1
    assert lib.etf_kv_free(None, 4096, 5, 4096, 1) == -1 and lib.etf_kv_take(h, None, 4096, 1, None, 4096, 4096, 4096, 4096, far) == -1
    for name in ("etf_kv_take_workspace_bytes", "etf_kv_fork_workspace_bytes", "etf_kv_compact_workspace_bytes"):
        more = (1,) if "take" in name else ()
        assert of(name, *more) > 0 and of(name, *more, batch=0) == -1
