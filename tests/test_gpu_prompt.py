"""Attention of packed prompts on the GPU against the oracle in float64 (oracle/prompt.py).

Bounds.  With u the type's rounding (half its epsilon) and e = 2^-24: a logit is a sum of D products that are exact in float32, so
it is off by at most delta = (D + 4) e mag, mag = sum_d |q_d k_d| scale; its exponential by 2 delta + 4 e (1 + reach).  A weight is
then rounded to the type (u), and sums of `seen` terms in float32 add seen * e of their absolute terms.  With size = sum p |v| that
makes out off by (u + 2 w) size + u |out|, w = 2 delta + 4 e (1 + reach) + seen e.  In float16 a weight below the type's normal
numbers is off by 2^-25 of the largest (seen 2^-25 vmax in all), the output by 2^-25.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import prompt  # noqa: E402
import paper_1509_05186_amd as etf  # noqa: E402

BF, HF = torch.bfloat16, torch.float16
E = 2.0 ** -24


def say(*a):
    print(*a, flush=True)


def context():
    return etf.Context(device=0, stream=torch.cuda.current_stream().cuda_stream)


def starts_of(lens, first=0):
    at = [first]
    for n in lens:
        at.append(at[-1] + n)
    return at


def rows(g, dtype, tokens, Hq, H, D, size=1.0):
    q = (size * torch.randn(tokens, Hq, D, generator=g)).to(dtype)
    k = (torch.randn(tokens, H, D, generator=g) + torch.randn(tokens // 32 + 1, H, D, generator=g).repeat_interleave(32, 0)[:tokens]).to(dtype)
    v = (torch.randn(tokens, H, D, generator=g) * torch.exp(torch.randn(1, H, 1, generator=g))).to(dtype)
    return q, k, v


def check(r, out, lse, dtype, what):
    u, D = torch.finfo(dtype).eps / 2, out.shape[-1]
    delta = (D + 4) * E * r["mag"]
    p = 2 * delta + 4 * E * (1 + r["reach"])
    w = (p + r["seen"] * E)[..., None]
    tol = (u + 2 * w) * r["size"] + u * r["out"].abs() + 1e-30
    if dtype == HF:
        tol += 2.0 ** -25 * r["seen"][..., None] * r["vmax"][..., None] + 2.0 ** -25
    some = ~torch.isnan(r["out"])
    out = out.double().cpu()
    assert not torch.isnan(out[some]).any(), what
    over = ((out - r["out"]).abs() / tol)[some]
    assert not over.numel() or float(over.max()) <= 1, "%s: out %.3g of its bound" % (what, float(over.max()))
    some = ~torch.isnan(r["lse"])
    off = (lse.double().cpu() - r["lse"]).abs()[some]
    tol = (p + r["seen"] * E + 4 * E * (1 + r["lse"].abs()))[some]
    assert (off <= tol).all(), "%s: lse %.3g of its bound" % (what, float((off / tol).max()))
    say("   out %.3f lse %.3f of their bounds" % (float(over.max()) if over.numel() else 0, float((off / tol).max()) if off.numel() else 0))


def run(q, k, v, starts, scale=None, ctx=None):
    """(out, lse); rows that the call leaves alone keep 7"""
    out, lse = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")
    got = (ctx or context()).prompt_attend(q.cuda(), k.cuda(), v.cuda(), torch.tensor(starts, dtype=torch.int32, device="cuda"), scale=scale, out=out, lse=lse)
    assert got is out
    torch.cuda.synchronize()
    return out, lse


def against_oracle(q, k, v, starts, what, scale=None):
    say(what)
    out, lse = run(q, k, v, starts, scale)
    r = prompt.attend(q, k, v, starts, q.shape[-1] ** -0.5 if scale is None else scale)
    check(r, out, lse, q.dtype, what)
    none = torch.isnan(r["lse"])
    assert (out.cpu()[none] == 7).all() and (lse.cpu()[none] == 7).all(), "%s: rows of no sequence" % what


@pytest.mark.parametrize("dtype,D,H,g", [(BF, 128, 2, 4), (HF, 96, 3, 5), (BF, 64, 1, 1), (HF, 128, 1, 7), (BF, 96, 2, 16), (HF, 64, 2, 3)])
@pytest.mark.parametrize("lens", [[1], [2], [63], [64, 65], [1, 0, 31, 0, 0, 33, 1], [127, 128, 129], [300, 5, 200]])
def test_prompts(dtype, D, H, g, lens):
    gen = torch.Generator().manual_seed(sum(lens) + D)
    q, k, v = rows(gen, dtype, sum(lens), H * g, H, D)
    against_oracle(q, k, v, starts_of(lens), "prompts %s D %d H %d g %d lens %s" % (dtype, D, H, g, lens))


@pytest.mark.parametrize("dtype,D,H,g,lens", [(BF, 128, 1, 1, [1000]), (HF, 64, 1, 2, [1500, 700]), (BF, 128, 2, 40, [70, 9]), (HF, 96, 1, 129, [40])])
def test_long_prompts_and_wide_groups(dtype, D, H, g, lens):
    gen = torch.Generator().manual_seed(5)
    q, k, v = rows(gen, dtype, sum(lens), H * g, H, D)
    against_oracle(q, k, v, starts_of(lens), "prompts %s D %d H %d g %d lens %s" % (dtype, D, H, g, lens))


@pytest.mark.parametrize("dtype,D,H,g,lens", [(BF, 128, 1, 1, [2100]), (HF, 64, 1, 2, [1500]), (HF, 96, 2, 1, [1700, 1300]), (BF, 64, 1, 3, [64 * 24]), (BF, 128, 1, 1, [1, 64 * 30 + 1])])
def test_ranges(dtype, D, H, g, lens):
    """Few tiles of long prompts: their blocks are cut into ranges, and joined."""
    gen = torch.Generator().manual_seed(6)
    q, k, v = rows(gen, dtype, sum(lens), H * g, H, D)
    assert etf.Context(device=None).prompt_attend_workspace_bytes(sum(lens), H * g, H, D, len(lens)) > 0
    against_oracle(q, k, v, starts_of(lens), "ranges %s D %d H %d g %d lens %s" % (dtype, D, H, g, lens))


def test_ranges_with_what_is_not_finite():
    say("ranges, not finite")
    gen = torch.Generator().manual_seed(7)
    q, k, v = rows(gen, BF, 1800, 1, 1, 64)
    clean, _ = run(q, k, v, [0, 1800])
    for where in (3, 600, 1799):
        for name, dims in (("v", [5]), ("k", list(range(64)))):
            x = dict(k=k.clone(), v=v.clone())
            x[name][where, 0, 5] = math.nan
            out, _ = run(q, x["k"], x["v"], [0, 1800])
            bad = torch.isnan(out.cpu())
            want = torch.zeros_like(bad)
            want[where:, :, dims] = True
            assert torch.equal(bad, want), (name, where)
            assert torch.equal(out.cpu()[~want], clean.cpu()[~want])


@pytest.mark.parametrize("batch", [1, 63, 64, 65, 128, 129, 200, 4097])
def test_many_sequences(batch):
    lens = [(7 * b) % 5 for b in range(batch)]
    gen = torch.Generator().manual_seed(batch)
    q, k, v = rows(gen, BF, sum(lens) + 1, 4, 2, 64)
    against_oracle(q, k, v, starts_of(lens), "batch %d" % batch)


def test_rows_of_no_sequence_stay():
    gen = torch.Generator().manual_seed(3)
    q, k, v = rows(gen, BF, 500, 8, 2, 128)
    against_oracle(q, k, v, [40, 140, 300], "tokens before and behind")
    against_oracle(q, k, v, [500, 500], "no tokens at all")
    against_oracle(q, k, v, [-5, 100, 1 << 30], "starts outside of the tokens")


@pytest.mark.parametrize("D", [64, 96, 128])
def test_strides(D):
    """Views of one projection, and rows of heads of their own."""
    gen = torch.Generator().manual_seed(D)
    H, g, lens = 2, 3, [100, 37, 161]
    T = sum(lens)
    fused = torch.randn(T, H * (g + 2) + 1, D + 8, generator=gen).to(BF).cuda()
    q, k, v = fused[:, : H * g, :D], fused[:, H * g : H * g + H, :D], fused[:, H * g + H : -1, :D]
    starts = torch.tensor(starts_of(lens), dtype=torch.int32, device="cuda")
    ctx = context()
    want = ctx.prompt_attend(q.contiguous(), k.contiguous(), v.contiguous(), starts)
    assert torch.equal(ctx.prompt_attend(q, k, v, starts), want)
    by_head = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)]
    assert torch.equal(ctx.prompt_attend(*by_head, starts), want)
    # one key and value for all heads
    one = k[:, :1].expand(T, H, D)
    assert torch.equal(ctx.prompt_attend(q, one, one, starts), ctx.prompt_attend(q, one.contiguous(), one.contiguous(), starts))
    r = prompt.attend(q.cpu(), k.cpu(), v.cpu(), starts.tolist(), D ** -0.5)
    check(r, want, r["lse"], BF, "strides")


@pytest.mark.parametrize("dtype", [BF, HF])
def test_large_and_small_logits(dtype):
    gen = torch.Generator().manual_seed(8)
    for size, scale in ((30.0, 1.0), (1e-3, 1e-3), (100.0, 30.0)):
        q, k, v = rows(gen, dtype, 200, 4, 2, 64, size)
        against_oracle(q, k, v, [0, 150, 200], "size %g scale %g %s" % (size, scale, dtype), scale)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_extremes(dtype):
    """The type's largest and smallest numbers: logits that float32 holds without fractions, values of full size."""
    top = torch.finfo(dtype).max if dtype == HF else 1e18
    gen = torch.Generator().manual_seed(9)
    q, k, v = rows(gen, dtype, 130, 4, 1, 64)
    v = (v.sign() * top).to(dtype)
    k[:, :, 0], q[:, :, 0] = 0, 0
    q[100:, :, 0], k[::3, :, 0] = 200.0, 200.0
    against_oracle(q, k, v, [0, 130], "extremes %s" % dtype)
    tiny = (torch.randn(130, 1, 64, generator=gen) * 2.0 ** -24).to(dtype)
    against_oracle(q, k, tiny, [0, 130], "tiny values %s" % dtype)


@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64), (BF, 96)])
@pytest.mark.parametrize("where", [0, 5, 63, 64, 100, 140])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_what_is_not_finite_stays_with_the_rows_that_see_it(dtype, D, where, what):
    say("not finite", dtype, D, where, what)
    gen = torch.Generator().manual_seed(where)
    starts = [0, 120, 150]
    q, k, v = rows(gen, dtype, 150, 6, 2, D)
    clean, clean_lse = run(q, k, v, starts)
    end = 120 if where < 120 else 150
    for name in ("q", "k", "v"):
        x = dict(q=q.clone(), k=k.clone(), v=v.clone())
        x[name][where, 1, 3] = what
        out, lse = run(x["q"], x["k"], x["v"], starts)
        heads = [1] if name == "q" else [3, 4, 5]
        touched = torch.zeros(150, 6, dtype=torch.bool)
        touched[where : where + 1 if name == "q" else end, heads] = True
        assert torch.equal(out.cpu()[~touched], clean.cpu()[~touched]) and torch.equal(lse.cpu()[~touched], clean_lse.cpu()[~touched]), name
        o = out.cpu()[touched].double()
        if name == "q" or (name == "k" and math.isnan(what)):
            assert torch.isnan(o).all(), name
        elif name == "v":
            bad = ~torch.isfinite(o)
            assert bad[:, 3].all() and (o[:, 3].isnan().all() if math.isnan(what) else (o[:, 3] == what).all()), name
            bad[:, 3] = False
            assert not bad.any(), name
        else:
            want, _ = prompt.attend_rowwise(x["q"], x["k"], x["v"], starts, D ** -0.5)
            assert torch.equal(torch.isnan(want[touched]), torch.isnan(o)), name


def test_every_key_infinitely_far():
    q, k = torch.ones(70, 1, 64, dtype=BF), torch.full((70, 1, 64), -math.inf, dtype=BF)
    out, lse = run(q, k, torch.ones(70, 1, 64, dtype=BF), [0, 70])
    assert torch.isnan(out).all() and not torch.isfinite(lse).any()


def test_the_same_twice_and_in_a_graph():
    say("graph")
    gen = torch.Generator().manual_seed(2)
    lens = [200, 3, 700]
    q, k, v = (x.cuda() for x in rows(gen, BF, sum(lens), 8, 2, 128))
    starts = torch.tensor(starts_of(lens), dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = etf.Context(device=0, stream=side.cuda_stream)
        want = ctx.prompt_attend(q, k, v, starts)
        out = torch.empty_like(q)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            ctx.prompt_attend(q, k, v, starts, out=out)
        for i in range(3):
            out.fill_(0)
            graph.replay()
            side.synchronize()
            assert torch.equal(out, want)
            starts.copy_(torch.tensor(starts_of([100, 300, 503] if i == 0 else lens), dtype=torch.int32))
            want = ctx.prompt_attend(q, k, v, starts)
            side.synchronize()


def test_another_current_stream():
    """A context's work runs on its stream, whichever is current."""
    gen = torch.Generator().manual_seed(4)
    q, k, v = (x.cuda() for x in rows(gen, HF, 300, 4, 4, 96))
    starts = torch.tensor([0, 300], dtype=torch.int32, device="cuda")
    want = context().prompt_attend(q, k, v, starts)
    torch.cuda.synchronize()
    ctx = context()
    with torch.cuda.stream(torch.cuda.Stream()):
        out = ctx.prompt_attend(q, k, v, starts)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_rows_beyond_2_to_the_32():
    """Many short prompts whose rows lie beyond 2^32 elements: the last ones as in a call of their own."""
    say("far rows")
    Hq, H, D, n, each = 32, 8, 128, 11_000, 96
    T = n * each
    assert T * Hq * D > 1 << 32
    q = torch.zeros(T, Hq, D, dtype=BF, device="cuda")
    k = torch.zeros(T, H, D, dtype=BF, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    last = 3 * each
    q[-last:] = torch.randn(last, Hq, D, generator=gen, device="cuda").to(BF)
    k[-last:] = torch.randn(last, H, D, generator=gen, device="cuda").to(BF)
    ctx = context()
    out = ctx.prompt_attend(q, k, k, torch.arange(0, T + 1, each, dtype=torch.int32, device="cuda"))
    want = ctx.prompt_attend(q[-last:].clone(), k[-last:].clone(), k[-last:].clone(), torch.arange(0, last + 1, each, dtype=torch.int32, device="cuda"))
    assert torch.equal(out[-last:], want) and not want.isnan().any() and (out[: each * 10] == 0).all()


def test_a_row_does_not_depend_on_the_rows_beside_it():
    """The same prompt alone, and among others."""
    say("alone and among others")
    gen = torch.Generator().manual_seed(13)
    q, k, v = (x.cuda() for x in rows(gen, HF, 700, 6, 2, 96))
    ctx = context()
    among = ctx.prompt_attend(q, k, v, torch.tensor([0, 37, 500, 700], dtype=torch.int32, device="cuda"))
    alone = ctx.prompt_attend(q[37:500].clone(), k[37:500].clone(), v[37:500].clone(), torch.tensor([0, 463], dtype=torch.int32, device="cuda"))
    assert torch.equal(among[37:500], alone)


def test_ranges_on_another_stream_and_in_a_graph():
    """With a workspace: the library's own on a stream that is not the current one, one taken while the graph is captured, and the caller's."""
    say("ranges, streams, graph")
    gen = torch.Generator().manual_seed(21)
    lens = [1500, 700]
    q, k, v = (x.cuda() for x in rows(gen, HF, sum(lens), 2, 1, 64))
    starts = torch.tensor(starts_of(lens), dtype=torch.int32, device="cuda")
    need = context().prompt_attend_workspace_bytes(sum(lens), 2, 1, 64, 2)
    assert need > 0
    want = context().prompt_attend(q, k, v, starts)
    torch.cuda.synchronize()
    ctx = context()
    with torch.cuda.stream(torch.cuda.Stream()):
        out = ctx.prompt_attend(q, k, v, starts)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = etf.Context(device=0, stream=side.cuda_stream)
        for room in (None, torch.empty(need + 256, dtype=torch.uint8, device="cuda")):
            out = torch.empty_like(q)
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                ctx.prompt_attend(q, k, v, starts, out=out, ws=room)
            for _ in range(3):
                out.fill_(0)
                graph.replay()
                eager = ctx.prompt_attend(q, k, v, starts)
                side.synchronize()
                assert torch.equal(out, want) and torch.equal(eager, want)


def test_two_calls_at_once():
    """Two contexts on streams of their own, with ranges and without."""
    say("two at once")
    gen = torch.Generator().manual_seed(22)
    work = []
    for lens, dtype, D in (([1500, 700], HF, 64), ([40, 0, 900], BF, 128)):
        x = [t.cuda() for t in rows(gen, dtype, sum(lens), 2, 1, D)] + [torch.tensor(starts_of(lens), dtype=torch.int32, device="cuda")]
        work.append((x, context().prompt_attend(*x)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    ctxs = [etf.Context(device=0, stream=s.cuda_stream) for s in streams]
    outs = []
    for _ in range(10):
        for (x, _), s, ctx in zip(work, streams, ctxs):
            with torch.cuda.stream(s):
                outs.append(ctx.prompt_attend(*x))
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        assert torch.equal(out, work[i % 2][1]), i


@pytest.mark.parametrize("dtype,D,T", [(BF, 64, 70_001), (HF, 128, 66_000)])
def test_one_long_prompt(dtype, D, T):
    """Tens of thousands of tokens: some rows of it, each over what it sees, in float64."""
    say("long", dtype, D, T)
    gen = torch.Generator().manual_seed(23)
    q, k, v = rows(gen, dtype, T, 2, 1, D)
    out, lse = run(q, k, v, [0, T])
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    at = [0, 1, 63, 64, 4095, 33_333, T - 66, T - 2, T - 1]
    r = {name: [] for name in ("out", "lse", "size", "reach", "mag", "seen", "vmax")}
    kk, vv, scale = k[:, 0].double(), v[:, 0].double(), D ** -0.5
    for i in at:
        s = q[i].double() @ kk[: i + 1].T * scale
        lse_i = torch.logsumexp(s, 1)
        p = torch.exp(s - lse_i[:, None])
        for name, x in (("out", p @ vv[: i + 1]), ("lse", lse_i), ("size", p @ vv[: i + 1].abs()), ("reach", s.abs().amax(1)),
                        ("mag", (q[i].double().abs() @ kk[: i + 1].abs().T * scale).amax(1)), ("seen", torch.full((2,), i + 1.0, dtype=torch.float64)),
                        ("vmax", vv[: i + 1].abs().max().expand(2))):
            r[name].append(x)
    check({name: torch.stack(x) for name, x in r.items()}, out.cpu()[at], lse.cpu()[at], dtype, "long")


def test_gradients_are_refused():
    gen = torch.Generator().manual_seed(14)
    q, k, v = (x.cuda() for x in rows(gen, BF, 10, 2, 2, 64))
    starts = torch.tensor([0, 10], dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="gradient"):
        context().prompt_attend(q.requires_grad_(), k, v, starts)
    with torch.no_grad():
        context().prompt_attend(q, k, v, starts)
