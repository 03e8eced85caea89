"""Adapters whose matrices, inputs or gradients hold infinities: results are the definition's infinities, with their signs, and NaN only
where the definition has NaN."""
import pytest
import torch

import clear_forms as F
import paper_1906_00148_amd as she
from test_gpu_clear_adapters import RAGGED, inputs

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16
INF = float("inf")
# one launch for a few tiles, two launches, odd widths, ranks of several chunks
SHAPES = [(64, 128, 8), (96, 520, 30), (128, 1000, 50), (77, 131, 12), (128, 264, 130)]


@pytest.fixture(scope="module")
def ctx():
    with she.Context(she.TOY, 20, 64) as c:
        yield c


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("K,N,r", SHAPES)
@pytest.mark.parametrize("base", [None, "same", "sums"])
def test_results(ctx, dtype, K, N, r, base):
    a = inputs(dtype, *RAGGED, 3, r, K, N)
    a["up"][0, r // 2, 5], a["up"][0, r - 1, 70], a["up"][2, 0, N - 1] = INF, -INF, INF
    a["up"][2, 1, N - 3], a["up"][2, 2, N - 3] = INF, -INF            # NaN or an infinity, by the hidden values' signs
    a["up"][2, 3, 9] = float("nan")
    a["down"][1, 0, 3] = -INF
    a["x"][120, 1] = INF
    if base:
        g = torch.Generator().manual_seed(4)
        a["base"] = torch.randn(163, N, generator=g).to(dtype).cuda() if base == "same" else torch.randint(-99, 99, (163, N), generator=g, dtype=torch.int32).cuda()
    want, bound = F.adapters(**a)
    assert torch.isinf(want).any() and torch.isnan(want).any() and torch.isfinite(want).any()
    F.check(ctx.adapters(**a), want, bound, dtype)
    if base == "same":
        F.check(ctx.adapters(**a, out=a["base"]), want, bound, dtype)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("K,N,r", SHAPES)
def test_gradients(ctx, dtype, K, N, r):
    """An infinity in x reaches a column of ddown and all of dup; one in dy dx's row, ddown's rows and a column of dup; one in down dx's
    column."""
    for name, at in (("x", (130, 7)), ("dy", (20, 11)), ("down", (2, 1, 6))):
        a = inputs(dtype, *RAGGED, 3, r, K, N)
        a["dy"] = torch.randn(163, N, generator=torch.Generator().manual_seed(9)).to(dtype).cuda()
        a[name][at] = -INF
        for got, (want, bound), what in zip(ctx.adapters_grad(**a), F.adapters_grad(**a), ("dx", "ddown", "dup")):
            F.check(got, want, bound, dtype, (name, what))


def test_many_tiles_of_an_adapter(ctx):
    """Sums that several workgroups share."""
    a = inputs(BF16, [0, 5000], [1], 2, 20, 72, 136)
    a["dy"] = torch.randn(5000, 136, generator=torch.Generator().manual_seed(9)).to(BF16).cuda()
    a["x"][4000, 3], a["x"][100, 3], a["x"][2300, 9] = INF, INF, -INF
    for got, (want, bound), what in zip(ctx.adapters_grad(**a), F.adapters_grad(**a), ("dx", "ddown", "dup")):
        F.check(got, want, bound, BF16, what)
