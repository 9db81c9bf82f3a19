"""Tensors that carry a tangent (forward-mode differentiation): the attention calls have no derivative, and refuse them instead of losing it."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
import torch.autograd.forward_ad as fw  # noqa: E402
from oracle import kvcache as kv  # noqa: E402
import paper_1509_05186_amd as etf  # noqa: E402

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_prompt_pages_refusals import prompt, taken  # noqa: E402

BF = torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    return etf.Context(device=None)


def calls(ctx):
    """(call, its tensors) of everything that takes queries, keys or values."""
    c = etf.KvCache(**kv.new_cache(2, 3, 64, 4, BF))
    q, k, v, st = prompt()
    rows, one = torch.zeros(2, 5, 3, 64, dtype=BF), torch.zeros(2, 5, 6, 64, dtype=BF)
    return [(lambda q, k, v: ctx.prompt_attend(q, k, v, st), (q, k, v)), (lambda k, v: ctx.kv_append_packed(c, k, v, st), (k, v)),
            (lambda k, v: ctx.kv_append(c, k, v), (rows, rows)), (lambda q: ctx.kv_attend(c, q), (one,))]


@pytest.mark.parametrize("i", range(4))
@pytest.mark.parametrize("grad", [True, False])
def test_a_tangent_is_refused(ctx, i, grad):
    call, tensors = calls(ctx)[i]
    for j in range(len(tensors)):
        with fw.dual_level(), torch.set_grad_enabled(grad):
            x = [fw.make_dual(t, torch.ones_like(t)) if j == y else t for y, t in enumerate(tensors)]
            with pytest.raises(ValueError, match="tangent"):
                call(*x)
            x[j] = x[j].detach()
            taken(call, *x)
            taken(call, *tensors)     # others of the same level go on


@pytest.mark.parametrize("i", range(4))
def test_gradients_are_refused_within_a_level_too(ctx, i):
    call, tensors = calls(ctx)[i]
    with fw.dual_level():
        with pytest.raises(ValueError, match="gradient"):
            call(*(t.clone().requires_grad_() for t in tensors))
        with torch.no_grad():
            taken(call, *(t.clone().requires_grad_() for t in tensors))
