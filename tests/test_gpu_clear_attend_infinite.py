"""Attention over values that are infinite where tokens attend to them: a result is infinite as the definition's is, and NaN only where infinities of both
signs meet (include/she_clear.h), by every kernel and walk."""
import pytest
import torch

import clear_forms as C
import clear_step_forms as F
import test_gpu_clear_attend as A
import test_gpu_clear_shared as S
from test_gpu_clear_shared import ctx  # noqa: F401
from test_gpu_clear_shared_walks import CALLS

pytestmark = pytest.mark.gpu
BF16, F16, INF = torch.bfloat16, torch.float16, float("inf")


def put(a, row, page, places):
    """Infinities of either sign and of both at elements of values that are attended to."""
    for i, u in enumerate(places):
        at = int(row[u // page])
        a["v_pages"][at, u % page, :, 2] = INF
        a["v_pages"][at, u % page, :, 5] = -INF
        a["v_pages"][at, u % page, :, 7] = INF if i % 2 else -INF


def check(got, want, bound, dtype, what):
    assert torch.isposinf(want).any() and torch.isneginf(want).any()
    C.check(got, want, bound, dtype, what)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("news,lengths,Hq,Hkv,D", [([1] * 5, [40, 1, 33, 300, 129], 8, 2, 64), ([1], [3000], 4, 1, 128), ([2, 3], [50, 700], 6, 2, 256), ([200], [500], 4, 1, 128),
                                                   ([300, 257], [2000, 900], 4, 1, 64)])
def test_attention_over_a_request_s_own_places(ctx, dtype, news, lengths, Hq, Hkv, D):  # noqa: F811
    a = A.inputs(dtype, news, lengths, Hq, Hkv, D, 16)
    for r, n in enumerate(lengths):
        put(a, a["table"][r], 16, [0] if n < 50 else [3, 17, n - news[r]])
    check(ctx.attend_pages(**a), *C.attend(**a), dtype, (news, lengths))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("name", ["few_64", "few_256", "few_cut_128", "tile_few_64", "tile_few_128", "tile_few_256", "tile_tile_64", "whole_few_64", "whole_64", "whole_cut_256"])
def test_attention_behind_a_prefix(ctx, dtype, name):  # noqa: F811
    _, heads, page, groups, before, after = CALLS[name]
    groups = [(n, [(min(t, 6), max(min(t, 6), own)) for t, own in rs]) for n, rs in groups] if name == "tile_tile_64" else groups
    a = S.inputs(dtype, groups, *heads, page, before, after)
    put(a, a["prefix_table"][0], page, [0, groups[0][0] // 2, groups[0][0] - 1])
    check(ctx.attend_shared(**a), *F.shared(**a), dtype, name)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("news,lengths", [([1] * 3, [60, 300, 129]), ([200, 100], [500, 300])])
def test_weights_that_are_small(ctx, dtype, news, lengths):  # noqa: F811
    """Down to 2^-60 of the largest, far below the smallest number of float16."""
    a = A.inputs(dtype, news, lengths, 8, 2, 64, 16, spread=7.0)
    for r, n in enumerate(lengths):
        put(a, a["table"][r], 16, [3, 17, n - news[r]])
    check(ctx.attend_pages(**a), *C.attend(**a), dtype, (news, lengths))
    a = S.inputs(dtype, [(700, [(news[0], n) for n in lengths]), (90, [(1, 5)])], 8, 2, 64, 16, spread=7.0)
    put(a, a["prefix_table"][0], 16, [0, 333, 699])
    check(ctx.attend_shared(**a), *F.shared(**a), dtype, (news, lengths))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("news,lengths", [([1] * 3, [60, 300, 129]), ([200, 100], [500, 300])])
def test_queries_and_values_that_are_nan(ctx, dtype, news, lengths):  # noqa: F811
    """They reach the rows and elements that they are in, and no others."""
    a = A.inputs(dtype, news, lengths, 8, 2, 64, 16)
    put(a, a["table"][0], 16, [2, 9])
    a["v_pages"][int(a["table"][1, 1]), 4, :, 11] = float("nan")
    a["q"][-1, 3, 1] = float("nan")
    want, bound = C.attend(**a)
    assert torch.isnan(want[-1, 3]).all() and not torch.isnan(want[-1, 2, :2]).any()
    check(ctx.attend_pages(**a), want, bound, dtype, (news, lengths))
