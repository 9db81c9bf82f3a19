"""Values of the type's largest size in the attention of packed prompts: sums of weighted values that float32 does not hold although their mean is a
number of the type, means that rounded weights put above it, and rows beside such rows.

Bounds as in test_gpu_prompt.py; a power of two that the weights are multiplied by changes no rounding, and what comes out above the type's largest number
becomes that one, which is nearer to a mean that does not exceed it."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_gpu_prompt import BF, HF, against_oracle, rows, run, say, starts_of  # noqa: E402

TOP = {BF: torch.finfo(BF).max, HF: torch.finfo(HF).max}
# whole tiles, and ranges that are joined
SHAPES = [(64, 2, 3, [130, 1, 300]), (96, 1, 5, [200]), (128, 2, 1, [2, 65, 129]), (128, 1, 1, [2100]), (64, 1, 2, [1500, 700])]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D,H,g,lens", SHAPES)
@pytest.mark.parametrize("signs", ["one", "two", "few"])
def test_values_of_the_largest_size(dtype, D, H, g, lens, signs):
    gen = torch.Generator().manual_seed(D + len(lens))
    q, k, v = rows(gen, dtype, sum(lens), H * g, H, D)
    top = torch.full_like(v, TOP[dtype])
    if signs == "two":
        top = torch.where(v < 0, -top, top)
    if signs == "few":      # among ordinary ones
        top = torch.where(torch.rand(v.shape[:2], generator=gen)[..., None] < 0.02, top, v)
    against_oracle(q, k, top, starts_of(lens), "largest values, signs %s, %s D %d lens %s" % (signs, dtype, D, lens))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("n", [3, 64, 200, 2100])
def test_weights_that_are_all_rounded_up(dtype, sign, n):
    """All but a row's first token have the same weight, a little above the middle of two of the type's numbers, and all values are the largest: the
    quotient of the sums is above the largest number by up to a rounding."""
    half = torch.finfo(dtype).eps / 4      # half a step of the numbers from 0.5 to 1
    q, k = torch.zeros(n, 1, 64, dtype=dtype), torch.zeros(n, 1, 64, dtype=dtype)
    q[:, :, 0], k[1:, :, 0] = 1, -1
    v = torch.full((n, 1, 64), sign * TOP[dtype], dtype=dtype)
    against_oracle(q, k, v, [0, n], "rounded up %s %d" % (dtype, n), -math.log(0.5 + 1.02 * half))


@pytest.mark.parametrize("D,H,g,lens", SHAPES)
def test_rows_beside_and_dimensions_beside(D, H, g, lens):
    """Rows that see no large value, and dimensions that have none, are as without them, to the last bit; infinities stay infinities."""
    say("beside large sums", D, lens)
    gen = torch.Generator().manual_seed(D)
    T = sum(lens)
    q, k, v = rows(gen, BF, T, H * g, H, D)
    v[:, :, 7] *= 2.0 ** -60
    starts = starts_of(lens)
    clean, clean_lse = run(q, k, v, starts)
    at = starts[-2] + lens[-1] // 2      # of the last sequence; the tokens from here on have large values in dimension 3
    large = v.clone()
    large[at:, :, 3] = TOP[BF]
    out, lse = run(q, k, large, starts)
    assert torch.equal(lse, clean_lse) and torch.isfinite(out).all()
    touched = torch.zeros(out.shape, dtype=torch.bool)
    touched[at:, :, 3] = True
    assert torch.equal(out.cpu()[~touched], clean.cpu()[~touched])
    for what in (math.inf, math.nan):
        large[T - 1, :, 4] = what
        out, lse = run(q, k, large, starts)
        assert torch.equal(lse, clean_lse)
        touched[T - 1, :, 4] = True
        assert torch.equal(out.cpu()[~touched], clean.cpu()[~touched])
        bad = out[T - 1, :, 4].isnan() if math.isnan(what) else out[T - 1, :, 4] == math.inf
        assert bad.all() and torch.isfinite(out[at:, :, 3]).all()


def test_rows_before_a_large_value_keep_the_smallest_numbers():
    """A tile that is worked out again for some of its rows: the others have their own results, small as they are."""
    say("small beside large")
    gen = torch.Generator().manual_seed(5)
    q, k, v = rows(gen, BF, 100, 2, 1, 64)
    v = v * 2.0 ** -110
    clean, _ = run(q, k, v, [0, 100])
    v[60:] = TOP[BF]
    out, _ = run(q, k, v, [0, 100])
    assert torch.equal(out[:60], clean[:60]) and (out[:60] != 0).any() and torch.isfinite(out).all()
