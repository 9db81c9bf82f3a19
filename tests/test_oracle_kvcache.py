"""The oracle of the attention cache against independent definitions, and the refusals of the calls etf_kv_* (no GPU)."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")
from oracle import kvcache as kv  # noqa: E402
import paper_1509_05186_amd as etf  # noqa: E402
from paper_1509_05186_amd import binding  # noqa: E402


def test_rounding_to_codes_is_the_types_own():
    x = torch.randn(20000, generator=torch.Generator().manual_seed(1)).double() * torch.exp2(torch.randint(-12, 7, (20000,), generator=torch.Generator().manual_seed(2)))
    x = torch.cat([x.clamp(-448, 448), torch.tensor([0.0, 448.0, -448.0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 1.0625, 1.1875])])
    assert torch.equal(kv.e4m3(x).float(), x.float().to(torch.float8_e4m3fn).float())
    assert [kv.scale_of(a) for a in (0, 448.0, 448.1, 1.0, 0.875, 0.876)] == [1.0, 1.0, 2.0, 2.0 ** -8, 2.0 ** -9, 2.0 ** -8]


def test_a_block_sealed_by_hand():
    c = kv.new_cache(1, 1, 64, 2, torch.bfloat16)
    k = torch.zeros(1, 64, 1, 64, dtype=torch.bfloat16)
    k[0, 3, 0, 5], k[0, 4, 0, 5], k[0, 9, 0, 0] = 900.0, -3.0, 2.0 ** -8
    kv.append(c, k, 2 * k)
    # 900 needs a scale of 4; 225 lies between 224 and 240; -3/4 is a code; 2^-10 is half the smallest code and goes to even
    assert c["scales"][0].tolist() == [4.0, 8.0]
    assert c["k"][0].float()[3, 5] == 224 and c["k"][0].float()[4, 5] == -0.75 and c["k"][0].float()[9, 0] == 0
    assert c["bounds"][0].float()[:, 5].tolist() == [-0.75, 224.0]
    assert c["v"][0].float()[5, 3] == 224


def test_tokens_come_out_the_same_whatever_pieces_they_came_in():
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(2, 300, 2, 64, generator=g).to(torch.float16) for _ in range(2))
    caches = []
    for piece in (300, 1, 77):
        c = kv.new_cache(2, 2, 64, 5, torch.float16)
        for i in range(0, 300, piece):
            kv.append(c, k[:, i : i + piece], v[:, i : i + piece])
            c["lens"] += min(piece, 300 - i)
        caches.append([kv.tokens(c, b, h) for b in range(2) for h in range(2)])
    for other in caches[1:]:
        for x, y in zip(caches[0], other):
            assert all(torch.equal(p, q) for p, q in zip(x, y))
    # within half a step of what went in, where it is a code, and itself where it is open still
    for b in range(2):
        for h in range(2):
            got, want = caches[0][2 * b + h][0], k[b, :, h].double()
            assert torch.equal(got[256:], want[256:])
            amax = want[:256].view(4, -1).abs().amax(1).repeat_interleave(64)[:, None]
            assert ((got - want)[:256].abs() <= torch.maximum(want[:256].abs() * 2.0 ** -4, amax * 2.0 ** -17)).all()


def test_attention_is_the_softmax_of_the_products():
    g = torch.Generator().manual_seed(4)
    c = kv.new_cache(1, 2, 64, 4, torch.bfloat16)
    k, v = (torch.randn(1, 200, 2, 64, generator=g).bfloat16() for _ in range(2))
    kv.append(c, k, v)
    c["lens"] += 200
    q = torch.randn(1, 70, 6, 64, generator=g).bfloat16()
    r = kv.attend(c, q, 0.125)
    kk, vv = (torch.stack([kv.tokens(c, 0, h)[i] for h in range(2)]).repeat_interleave(3, 0) for i in (0, 1))
    s = q[0].transpose(0, 1).double() @ kk.transpose(1, 2) * 0.125
    s = s.masked_fill(torch.arange(200) > torch.arange(130, 200)[:, None], -math.inf)
    p = torch.softmax(s, -1)
    torch.testing.assert_close(r["out"][0], (p @ vv).transpose(0, 1), rtol=1e-12, atol=1e-12)
    torch.testing.assert_close(r["lse"][0], torch.logsumexp(s, -1).T, rtol=1e-12, atol=1e-12)
    per = torch.nn.functional.pad(p.view(2, 3, 70, 200).sum((1, 2)), (0, 56)).view(2, 4, 64).sum(-1)
    torch.testing.assert_close(r["mass"][0], per, rtol=1e-12, atol=1e-12)
    # all blocks listed is no list
    lists = torch.arange(4, dtype=torch.int32).expand(1, 70, 2, 4)
    assert torch.equal(kv.attend(c, q, 0.125, lists=lists)["out"], r["out"])
    # the score is a bound of every logit, and the chosen blocks are those of the largest scores
    lists = kv.select(c, q[:, -1:], 2, 0, 0)
    for h in range(2):
        score = []
        for j in range(3):
            b = c["bounds"][h * 4 + j].double() * float(c["scales"][h * 4 + j, 0])
            top = torch.maximum(q[0, -1, 3 * h : 3 * h + 3].double()[:, None] * b[0], q[0, -1, 3 * h : 3 * h + 3].double()[:, None] * b[1])
            score.append(float(top.sum(-1).sum(-1).max()))
            assert score[-1] >= float((q[0, -1, 3 * h : 3 * h + 3].double() @ kk[3 * h, 64 * j : 64 * j + 64].T).max())
        assert lists[0, 0, h].tolist() == sorted(sorted(range(3), key=lambda j: -score[j])[:2])


def test_eviction_by_hand():
    c = kv.new_cache(1, 1, 64, 7, torch.bfloat16)
    c["lens"][0], c["evicted"][0] = 6 * 64 + 10, 3
    mass = torch.tensor([[[1.0, 9.0, 5.0, 5.0, 0.0, 2.0, 0.5]]])
    table, lens, evicted, kept, freed = kv.evict(c, mass, 4, 1, 1)
    assert table[0, 0].tolist() == [0, 1, 2, 5, -1, -1, -1] and freed[0, 0].tolist() == [3, 4, -1, -1, -1, -1, -1]
    assert kept[0, 0].tolist() == [1.0, 9.0, 5.0, 2.0, 0.5, 0.0, 0.0] and lens.tolist() == [4 * 64 + 10] and evicted.tolist() == [5]


# ---- refusals: the library checks every argument before it asks for a GPU


def fake_cache(**over):
    c = binding.EtfKvCache(0, 2, 4, 64, 8, 100)
    for name in etf.KvCache.FIELDS:
        setattr(c, name, 4096)
    for name, value in over.items():
        setattr(c, name, value)
    return c


def strides(*s):
    return (ctypes.c_int64 * 3)(*s)


@pytest.fixture(scope="module")
def host():
    return etf.Context(device=None)


BAD_CACHES = [dict(dtype=2), dict(dtype=-1), dict(head_dim=32), dict(head_dim=80), dict(head_dim=0), dict(batch=0), dict(heads=-1), dict(max_blocks=0),
              dict(pages=0), dict(batch=1 << 20, heads=1 << 10, max_blocks=1 << 10), dict(max_blocks=1 << 26)]


@pytest.mark.parametrize("over", BAD_CACHES, ids=str)
def test_caches_that_are_refused(host, over):
    lib, h, c = host._lib, host._h, fake_cache(**over)
    r = ctypes.addressof(c)
    assert lib.etf_kv_append(h, r, 4096, None, 4096, None, 1, None) == -1
    assert lib.etf_kv_attend_workspace_bytes(h, r, 1, 8, 0, 0) == -1
    assert lib.etf_kv_attend(h, r, 4096, None, 1, 8, 1.0, None, None, 0, 4096, None, None, None, 4096, 1 << 40) == -1
    assert lib.etf_kv_select_workspace_bytes(h, r, 1, 8, 2) == -1
    assert lib.etf_kv_select(h, r, 4096, None, 1, 8, None, 2, 0, 0, 4096, 4096, 1 << 40) == -1
    assert lib.etf_kv_evict(h, r, 4096, 4, 1, 1, 4096, 4096, 4096, 4096, 4096) == -1


@pytest.mark.parametrize("name", etf.KvCache.FIELDS)
def test_arrays_that_are_refused(host, name):
    for value in (None, 4104):
        r = ctypes.addressof(fake := fake_cache(**{name: value}))
        assert host._lib.etf_kv_append(host._h, r, 4096, None, 4096, None, 1, None) == -1
        assert host._lib.etf_kv_attend(host._h, r, 4096, None, 1, 8, 1.0, None, None, 0, 4096, None, None, None, 4096, 1 << 40) == -1
        assert host._lib.etf_kv_select(host._h, r, 4096, None, 1, 8, None, 2, 0, 0, 4096, 4096, 1 << 40) == -1
        assert host._lib.etf_kv_evict(host._h, r, 4096, 4, 1, 1, 4096, 4096, 4096, 4096, 4096) == -1
        del fake


def test_arguments_that_are_refused(host):
    lib, h, c = host._lib, host._h, fake_cache()
    r = ctypes.addressof(c)

    def append(k=4096, ks=None, v=4096, vs=None, n=1, cache=r):
        return lib.etf_kv_append(h, cache, k, ks, v, vs, n, None)

    assert append() == -5                                   # everything right: a GPU is what is missing
    assert append(ks=strides(64 * 4 * 8, 64 * 4, 64)) == -5
    for bad in (dict(cache=None), dict(k=None), dict(v=None), dict(k=4104), dict(n=0), dict(n=-1), dict(n=(1 << 24) + 1), dict(ks=strides(1024, 260, 64)),
                dict(vs=strides(1024, 256, -64)), dict(vs=strides(1 << 41, 256, 64))):
        assert append(**bad) == -1, bad

    def attend(q=4096, qs=None, n=1, hq=8, scale=1.0, lists=None, w=0, out=4096, mass_in=None, mass_out=None, ws=4096, nbytes=1 << 40):
        return lib.etf_kv_attend(h, r, q, qs, n, hq, scale, None, lists, w, out, None, mass_in, mass_out, ws, nbytes)

    assert attend() == -5 and attend(lists=4096, w=3) == -5 and attend(mass_in=4096, mass_out=4096) == -5
    for bad in (dict(q=None), dict(q=4100), dict(n=0), dict(hq=0), dict(hq=6), dict(n=1 << 26), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf),
                dict(scale=math.nan), dict(w=3), dict(lists=4096), dict(lists=4096, w=4097), dict(lists=4096, w=3, mass_out=4096), dict(mass_in=4096),
                dict(out=None), dict(out=4100), dict(ws=None), dict(ws=4100), dict(qs=strides(8, 7, 8))):
        assert attend(**bad) == -1, bad
    need = lib.etf_kv_attend_workspace_bytes(h, r, 1, 8, 0, 1)
    assert need > 0 and attend(mass_out=4096, nbytes=need - 1) == -3 and b"workspace too small" in lib.etf_last_error(h)
    assert attend(mass_out=4096, nbytes=need) == -5
    for n, hq, w, mass in ((0, 8, 0, 0), (1, 7, 0, 0), (1, 8, -1, 0), (1, 8, 4097, 0), (1, 8, 2, 1)):
        assert lib.etf_kv_attend_workspace_bytes(h, r, n, hq, w, mass) == -1

    def select(q=4096, n=1, hq=8, w=4, sink=1, recent=1, lists=4096, ws=4096, nbytes=1 << 40):
        return lib.etf_kv_select(h, r, q, None, n, hq, None, w, sink, recent, lists, ws, nbytes)

    assert select() == -5 and select(w=1, sink=1, recent=0) == -5
    for bad in (dict(q=None), dict(n=0), dict(hq=5), dict(w=0), dict(w=4097), dict(sink=-1), dict(recent=-1), dict(sink=3, recent=2),
                dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1), dict(lists=None), dict(ws=None), dict(ws=4104)):
        assert select(**bad) == -1, bad
    need = lib.etf_kv_select_workspace_bytes(h, r, 1, 8, 4)
    assert need > 0 and select(nbytes=need - 1) == -3 and select(nbytes=need) == -5

    def evict(mass=4096, budget=4, sink=1, recent=1, table=4096, lens=4096, evicted=4096, out=4096, freed=4096):
        return lib.etf_kv_evict(h, r, mass, budget, sink, recent, table, lens, evicted, out, freed)

    assert evict() == -5
    for bad in (dict(mass=None), dict(budget=0), dict(sink=-1), dict(recent=-2), dict(sink=3, recent=2), dict(table=None), dict(lens=None), dict(evicted=None),
                dict(out=None), dict(freed=None)):
        assert evict(**bad) == -1, bad
    c.max_blocks = 16385                                    # too long a row to be cut in place
    assert evict() == -1 and evict(table=8192) == -1 and evict(table=8192, out=8192) == -5
    c.max_blocks = 16384
    assert evict() == -5
    c.max_blocks = 8


def test_the_bindings_checks():
    def cache(**over):
        t = dict(kv.new_cache(2, 3, 64, 4, torch.bfloat16), **over)
        return etf.KvCache(**t)

    c, ctx = cache(), etf.Context(device=None)
    for over in (dict(k=torch.zeros(24, 64, 64)), dict(v=torch.zeros(23, 64, 64).to(torch.float8_e4m3fn)), dict(lens=torch.zeros(2, dtype=torch.int64)),
                 dict(table=torch.zeros(2, 4, 3, dtype=torch.int32)), dict(tail_k=torch.zeros(2, 3, 2, 64, 64)), dict(table=torch.zeros(2, 3, 4, 2, dtype=torch.int32)),
                 dict(tail_v=torch.zeros(2, 3, 2, 64, 64, dtype=torch.bfloat16).transpose(-1, -2))):
        with pytest.raises(ValueError):
            cache(**over)
    q = torch.zeros(2, 1, 6, 64, dtype=torch.bfloat16)
    ws = torch.empty(ctx.kv_attend_workspace_bytes(c, 1, 6) + 256, dtype=torch.uint8)
    out = torch.empty_like(q)
    with pytest.raises(etf.EtfError) as e:
        ctx.kv_attend(c, q, out=out, ws=ws)
    assert e.value.code == -5
    for bad in (q[:1], q[0], q.half(), q[..., :32], q.transpose(2, 3)):
        with pytest.raises(ValueError):
            ctx.kv_attend(c, bad, out=out, ws=ws)
        with pytest.raises(ValueError):
            ctx.kv_select(c, bad, 2, ws=ws)
    with pytest.raises(ValueError):
        ctx.kv_append(c, q[:, :, :3], q[:, :, :2])
    with pytest.raises(ValueError):
        ctx.kv_append(c, q[:, :, :3], torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16))
    for bad in (dict(counts=torch.zeros(2)), dict(counts=torch.zeros(3, dtype=torch.int32)), dict(lists=torch.zeros(2, 1, 6, 2, dtype=torch.int32)),
                dict(lse=torch.zeros(2, 1, 5)), dict(mass_out=torch.zeros(2, 3, 5)), dict(out=torch.empty(2, 1, 6, 64))):
        with pytest.raises(ValueError):
            ctx.kv_attend(c, q, **{**dict(out=out, ws=ws), **bad})
    with pytest.raises(ValueError):
        ctx.kv_evict(c, torch.zeros(2, 3, 3), 2)
    assert not hasattr(c, "nonsense") and c.fork().k is c.k and c.fork().lens is not c.lens
