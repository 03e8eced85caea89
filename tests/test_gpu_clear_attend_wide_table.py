"""Attention for single tokens through tables much wider than most requests need, as a serving program keeps them: a request that does
fill its table has pieces longer than the places that are looked up together.  Against the definition in 64 bits."""
import pytest
import torch

import paper_1906_00148_amd as she
from test_gpu_clear_attend import compare, inputs

pytestmark = pytest.mark.gpu
REQUESTS, HEADS, PAGE = 136, 8, 64
LENGTHS = [(37 * i) % 300 + 1 for i in range(REQUESTS)]
LENGTHS[5], LENGTHS[77], LENGTHS[130] = 17000, 40001, 16385


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
    """Places 3000 and 7000 of the long request's first pieces, and its last places."""
    a = inputs(torch.bfloat16, [1] * REQUESTS, LENGTHS, HEADS, HEADS, 64, PAGE)
    a["table"][77, 3000 // PAGE] = -1
    ctx.clear_bad_ids()
    compare(ctx, a, torch.bfloat16)
    assert ctx.clear_bad_ids() > 0
    # with a window the places before it are not attended to, whatever they hold
    a["v_pages"][int(a["table"][77, 15])] = float("nan")          # places 960 to 1023, and up to 1030 of the first 32 that are read
    a["v_pages"][int(a["table"][77, 16]), :7] = float("nan")
    compare(ctx, a, torch.bfloat16, 40001 - 1031)
