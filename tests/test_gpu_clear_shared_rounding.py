"""Attention behind shared prefixes for requests of few rows, whose prefixes go by tiles of many rows: a result's error is that of its own rounding."""
import pytest
import torch

import clear_forms as C
import clear_step_forms as F
from test_gpu_clear_shared import ctx, inputs  # noqa: F401

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16
# heads, page, prefixes with their requests, window
CALLS = {
    "single_tokens": ((8, 1, 128), 64, [(4000, [(1, 1 + 7 * n % 90) for n in range(64)])], 0),
    "heads_of_64": ((8, 2, 64), 16, [(2000, [(1, 1 + 3 * n % 50) for n in range(60)]), (700, [(1, 3)] * 30)], 0),
    "heads_of_192": ((6, 1, 192), 16, [(1500, [(1, 1 + 3 * n % 50) for n in range(60)])], 0),
    "few_tokens": ((16, 16, 64), 16, [(1800, [(1 + n % 4, 4 + 11 * n % 300) for n in range(40)])], 0),
    "a_window": ((28, 4, 80), 24, [(2500, [(1 + n % 2, 600 + n) for n in range(20)]), (1700, [(2, 800)] * 13)], 2048),
    "rows_of_a_wavefront": ((8, 1, 64), 16, [(1500, [(3, 300 + n) for n in range(24)])], 0),
}


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("name", CALLS)
def test_nothing_but_the_result_s_own_rounding(ctx, name, dtype):  # noqa: F811
    heads, page, groups, window = CALLS[name]
    a = inputs(dtype, groups, *heads, page)
    got = ctx.attend_shared(**a, window=window).double().cpu()
    want, bound = F.shared(**a, window=window)
    # the bound has a weight's rounding to the type, a unit of the weighted sizes of the values: of two numbers only what they leave counts
    sizes, _ = F.shared(**dict(a, v_pages=a["v_pages"].abs()), window=window)
    bound = bound - (C.UNIT[dtype] - C.SPLIT[dtype]) * sizes
    assert bool((bound >= 0).all())
    off = (got - want).abs()
    assert bool((off <= C.UNIT[dtype] * want.abs() + C.TINY[dtype] + bound).all()), float((off / (C.UNIT[dtype] * want.abs() + C.TINY[dtype] + bound)).max())
