"""Attention behind shared prefixes: calls that go every way that the host chooses from (csrc/clear_attend_shape.cpp): prefixes by tiles of
few or many rows, what the requests have behind them likewise, or both as one walk, cut or not.  tests/test_host_clear_shared_shapes.py
holds each call to its way."""
import pytest
import torch

import test_gpu_clear_shared as S
from test_gpu_clear_shared import compare, ctx, inputs  # noqa: F401

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16

# way: prefix walk (or both as one), own walk, whether the pieces of the own walk (or of the one walk) are several
# name -> (way, heads, page, groups, requests before and after them)
CALLS = {
    "few_64": (("few", "few", False), (8, 2, 64), 16, [(600, [(1, n) for n in range(1, 20)]), (0, [(2, 2)])], [(1, 7)], [(3, 5)]),
    "few_128": (("few", "few", False), (4, 4, 128), 1, [(533, [(1, n) for n in range(1, 20)])], [], [(1, 9)]),
    "few_256": (("few", "few", False), (6, 2, 256), 24, [(400, [(1, n) for n in range(1, 20)])], [(4, 4)], []),
    "few_cut_64": (("few", "few", True), (2, 2, 64), 16, [(600, [(1, 900), (2, 1500), (1, 3)])], [], []),
    "few_cut_128": (("few", "few", True), (4, 1, 96), 16, [(600, [(1, 900), (2, 1500), (1, 3)]), (50, [(1, 600)])], [(1, 800)], []),
    "few_cut_256": (("few", "few", True), (3, 1, 192), 16, [(600, [(1, 900), (2, 1500), (1, 3)])], [], [(1, 1)]),
    "tile_few_64": (("tile", "few", False), (8, 2, 64), 16, [(2000, [(1, 1 + 3 * n % 50) for n in range(60)]), (700, [(1, 3)] * 30)], [], [(1, 30)]),
    "tile_few_128": (("tile", "few", False), (8, 1, 128), 24, [(1500, [(1, 1 + 3 * n % 50) for n in range(60)])], [(2, 9)], []),
    "tile_few_80": (("tile", "few", False), (14, 2, 80), 5, [(1211, [(1, 1 + 3 * n % 50) for n in range(60)])], [], []),
    "tile_few_256": (("tile", "few", False), (8, 1, 256), 16, [(1500, [(1, 1 + 3 * n % 50) for n in range(50)])], [], []),
    "tile_few_cut_64": (("tile", "few", True), (4, 1, 64), 16, [(3000, [(1, 500)] + [(2, 30)] * 40)], [], []),
    "tile_few_cut_128": (("tile", "few", True), (4, 1, 128), 16, [(3000, [(1, 500)] + [(2, 30)] * 40)], [], []),
    "tile_few_cut_256": (("tile", "few", True), (4, 1, 256), 16, [(3000, [(1, 500)] + [(2, 30)] * 40)], [], []),
    "tile_tile_64": (("tile", "tile", False), (8, 2, 64), 16, [(2000, [(90, 400), (1, 300), (70, 70), (130, 390), (0, 8), (20, 300)])], [(1, 40)], [(33, 40)]),
    "tile_tile_128": (("tile", "tile", False), (8, 1, 96), 64, [(2000, [(90, 400), (1, 300), (70, 70), (60, 390), (0, 8), (20, 300)]), (100, [(20, 40)])], [], []),
    "tile_tile_cut_64": (("tile", "tile", True), (8, 1, 64), 16, [(1200, [(40, 1500), (30, 900), (35, 40), (1, 1200), (50, 1300)])], [], [(5, 1200)]),
    "tile_tile_cut_128": (("tile", "tile", True), (8, 1, 128), 16, [(1200, [(40, 1500), (30, 900), (35, 40), (1, 1200)])], [(20, 700)], []),
    "whole_few_64": (("whole", "few", False), (8, 2, 64), 16, [(300, [(1, n) for n in range(1, 20)]), (0, [(2, 2)]), (77, [(5, 9), (1, 100)])], [(1, 7)], [(3, 5)]),
    "whole_few_128": (("whole", "few", False), (4, 4, 128), 1, [(333, [(1, n) for n in range(1, 20)]), (40, [(7, 7)])], [(6, 50)], [(1, 9)]),
    "whole_few_80": (("whole", "few", False), (12, 2, 80), 24, [(200, [(1, 130), (9, 99)])], [], []),
    "whole_few_256": (("whole", "few", False), (6, 2, 256), 24, [(250, [(1, n) for n in range(1, 20)]), (9, [(6, 12)])], [(4, 4)], []),
    "whole_64": (("whole", "tile", False), (16, 1, 64), 16, [(200, [(150, 160), (100, 101), (9, 150), (120, 130)]), (0, [(60, 90)])], [(50, 90)], [(3, 5)]),
    "whole_128": (("whole", "tile", False), (16, 1, 128), 24, [(200, [(150, 160), (100, 101), (9, 150), (120, 130)]), (77, [(60, 90)])], [], [(50, 60)]),
    "whole_cut_256": (("whole", "tile", True), (12, 2, 256), 16, [(900, [(60, 400), (1, 200), (35, 35), (50, 390)]), (333, [(20, 60)])], [(9, 200)], [(3, 50)]),
    "whole_cut_192": (("whole", "tile", True), (8, 1, 192), 5, [(700, [(30, 300), (1, 200), (35, 35), (50, 290)])], [], []),
}


def shapes():
    """For each call: what tests/host_checks/shared_shape.cpp reads."""
    got = {}
    for name, (_, (Hq, Hkv, D), page, groups, before, after) in CALLS.items():
        requests = [*before, *(r for _, rs in groups for r in rs), *after]
        width = [max([-(-n // page) for n in some] + [1]) for some in ([n for n, _ in groups], [n for _, n in requests])]
        got[name] = (sum(n for n, _ in requests), len(requests), Hq, Hkv, D, 0, len(groups), *width, page)
    return got


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("name", CALLS)
def test_every_way(ctx, name, dtype):  # noqa: F811
    _, heads, page, groups, before, after = CALLS[name]
    a = inputs(dtype, groups, *heads, page, before, after)
    for window in (0, 1, 130, 700):
        if shapes()[name][0] * heads[0] < 20000 or window in (0, 700):
            got = compare(ctx, a, dtype, window, (name, window))
            assert torch.equal(got, ctx.attend_shared(**a, window=window))


@pytest.mark.parametrize("name", CALLS)
def test_every_way_with_places_that_are_not_there(ctx, name):  # noqa: F811
    """Page ids out of range, tables short of a column, own lengths short of the new tokens, prefixes shorter than their table."""
    _, heads, page, groups, before, after = CALLS[name]
    a = inputs(BF16, groups, *heads, page, before, after, spread=3.0)
    a["prefix_table"][0, 1], a["table"][len(before), -1] = -3, 1 << 30
    a["prefix_lengths"][0] -= page // 2 + 1
    a["lengths"][len(before)] = max(0, int(a["starts"][len(before) + 1] - a["starts"][len(before)]) - 1)
    ctx.clear_bad_ids()
    for window in (0, 250):
        compare(ctx, a, BF16, window, (name, window))
    assert ctx.clear_bad_ids() > 0
    short = dict(a, prefix_table=a["prefix_table"][:, :-1].contiguous(), table=a["table"][:, :-1].contiguous())
    for window in (0, 250):
        compare(ctx, short, BF16, window, (name, window))


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("special", [float("inf"), float("nan")])
def test_every_way_with_values_that_are_not_finite_where_a_window_hides_them(ctx, name, special):  # noqa: F811
    """The window of the prefix's readers begins behind such places for some of a tile's rows and before them for others."""
    _, heads, page, groups, before, after = CALLS[name]
    a = inputs(F16, groups, *heads, page, before, after)
    P = groups[0][0]
    for u in (P - 30, P - 3, P // 2):
        at = int(a["prefix_table"][0, u // page])
        a["v_pages"][at, u % page, :, 1::3] = special
    window = 40
    want, bound = S.F.shared(**a, window=window)
    got = ctx.attend_shared(**a, window=window).double().cpu()
    fine = torch.isfinite(want) & torch.isfinite(bound)
    assert fine.any() and torch.equal(torch.isfinite(got), torch.isfinite(want))
    off = (got - want).abs()[fine]
    assert bool((off <= (bound + S.C.UNIT[F16] * want.abs() + S.C.TINY[F16])[fine]).all())
