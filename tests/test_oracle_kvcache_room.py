"""The oracle of the attention cache where a table is full: what it holds does not depend on the pieces in which its tokens came (no GPU)."""
import pytest

torch = pytest.importorskip("torch")
from oracle import kvcache as kv  # noqa: E402


@pytest.mark.parametrize("total", [128, 190, 191, 192, 300])
def test_tokens_past_the_tables_end_are_dropped_and_the_others_kept(total):
    """Two blocks and the 63 tokens of an open one: 191 tokens are counted, and those are written."""
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(1, total, 1, 64, generator=g).to(torch.float16) for _ in range(2))
    held = min(total, 191)
    for piece in (1, 60, 77, 130, 300):
        c = kv.new_cache(1, 1, 64, 2, torch.float16)
        c["tail_k"].fill_(float("nan"))
        for i in range(0, total, piece):
            kv.append(c, k[:, i : i + piece], v[:, i : i + piece])
            c["lens"] += min(piece, total - i)
        got, values, there = kv.tokens(c, 0, 0)
        assert got.shape[0] == held and there.all()
        assert torch.equal(got[128:], k[0, 128:held, 0].double()) and torch.equal(values[128:], v[0, 128:held, 0].double())
