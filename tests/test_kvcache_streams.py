"""Which stream the cache calls' own allocations belong to: the context's, whatever stream is the program's (no GPU: torch's streams are stood in for)."""
import contextlib

import pytest

torch = pytest.importorskip("torch")
from oracle import kvcache as kv  # noqa: E402
import paper_1509_05186_amd as etf  # noqa: E402
from paper_1509_05186_amd import binding  # noqa: E402


@pytest.mark.parametrize("own,program", [(None, 77), (0, 77), (5, 77), (5, 0), (77, 77), (None, 0)])
def test_allocations_are_made_on_the_contexts_stream(monkeypatch, own, program):
    now = [program]

    @contextlib.contextmanager
    def stream(s):
        now.append(s)
        yield
        now.pop()

    def external(pointer, device=None):
        assert pointer, "torch takes a stream of its pool for a pointer of zero"
        return pointer

    monkeypatch.setattr(binding, "_current_stream", lambda gpu: now[-1])
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", external)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: 0)
    made, empty = [], torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: made.append(now[-1]) or empty(*a, **k))
    ctx, c = etf.Context(device=None), etf.KvCache(**kv.new_cache(2, 3, 64, 4, torch.bfloat16))
    ctx._stream = own
    ctx._kv_empty((3,), torch.int32, c)
    ctx._kv_scratch(c, etf.Context.kv_select_workspace_bytes, 1, 6, 2)
    assert made and all(s == (own or 0) for s in made) and now == [program]
