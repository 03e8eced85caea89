"""Attention for single tokens through tables much wider than most requests need, as a serving program keeps them: a request that does
fill its table has pieces longer than the places that are looked up together.  Against the definition in 64 bits."""
import pytest
import torch

import paper_1906_00148_amd as she
from test_gpu_clear_attend import compare, inputs

pytestmark = pytest.mark.gpu
REQUESTS, HEADS, PAGE = 136, 8, 64
LENGTHS = [(37 * i) % 300 + 1 for i in range(REQUESTS)]
LENGTHS[5], LENGTHS[77], LENGTHS[130] = 31000, 40001, 16385


@pytest.fixture(scope="module")
def ctx():
    with she.Context(she.TOY, 16, 64) as c:
        yield c


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("window", [0, 39000])
def test_long_requests_among_short_ones(ctx, dtype, window):
    a = inputs(dtype, [1] * REQUESTS, LENGTHS, HEADS, HEADS, 64, PAGE)
    got = compare(ctx, a, dtype, window)
    wide = torch.full((REQUESTS, 131072 // PAGE), -1, dtype=torch.int32, device="cuda")
    wide[:, :a["table"].shape[1]] = a["table"]
    compare(ctx, dict(a, table=wide), dtype, window)
    assert torch.equal(got, ctx.attend_pages(**a, window=window))


def test_what_is_missing_or_not_finite_in_a_later_block(ctx):
    """Places after the 2048 that are looked up first, in the first piece of the long request and in the third."""
    a = inputs(torch.bfloat16, [1] * REQUESTS, LENGTHS, HEADS, HEADS, 64, PAGE)
    a["table"][77, 2500 // PAGE] = a["table"][77, 7600 // PAGE] = -1
    ctx.clear_bad_ids()
    compare(ctx, a, torch.bfloat16)
    assert ctx.clear_bad_ids() > 0
    # with a window the places before it are not attended to, whatever they hold
    a["v_pages"][int(a["table"][77, 15])] = float("nan")          # places 960 to 1023, and up to 1030 of the first 32 that are read
    a["v_pages"][int(a["table"][77, 16]), :7] = float("nan")
    compare(ctx, a, torch.bfloat16, 40001 - 1031)


@pytest.mark.parametrize("page", [1, 16, 24])
@pytest.mark.parametrize("news,lengths,heads,window", [([1, 1], [700, 95], (4, 2), 50), ([3, 1], [700, 96], (4, 2), 60), ([700, 800], [1000, 1333], (8, 1), 75)])
def test_pages_that_a_window_has_passed_may_be_gone(ctx, page, news, lengths, heads, window):
    """A cache that gives back the pages that no token of a window reaches, as soon as it can: none of their ids is counted, the first one
    that a token does reach is.  Single tokens, a few, and many (the kernel for tiles of rows)."""
    a = inputs(torch.bfloat16, news, lengths, *heads, 64, page)
    want = ctx.attend_pages(**a, window=window)
    first = [max(0, length - n - window + 1) // page for n, length in zip(news, lengths)]       # the first page that is needed
    for r, n in enumerate(first):
        a["table"][r, :n] = -1
    ctx.clear_bad_ids()
    assert torch.equal(ctx.attend_pages(**a, window=window), want) and ctx.clear_bad_ids() == 0
    a["table"][0, first[0]] = -1
    compare(ctx, a, torch.bfloat16, window)
    assert ctx.clear_bad_ids() > 0
