"""Attention over a paged cache where a call has many rows: the kernel for tiles of them, at masks, tables and sizes where it can go wrong,
against the definition in 64 bits.  tests/test_host_clear_shapes.py checks that these calls are that kernel's."""
import pytest
import torch

import clear_forms as F
import paper_1906_00148_amd as she
from test_gpu_clear_attend import compare, inputs

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    with she.Context(she.TOY, 15, 64) as c:
        yield c


# tokens and lengths of each request, heads, page, the table's columns, window
BEYOND_THE_TABLE = [([2048], [2048], 1, 1, 64, 16, 17, 0), ([300], [2000], 4, 1, 128, 16, 65, 0), ([500, 1, 300], [1100, 1500, 400], 4, 2, 64, 24, 43, 0),
                    ([600, 200], [900, 700], 2, 1, 96, 1, 777, 700), ([400], [1300], 4, 1, 256, 16, 67, 0)]
# heads, and page and window; tokens and lengths of the requests
HEADS = [(16, 2, 64), (8, 1, 128), (12, 1, 80), (7, 1, 192), (8, 1, 256)]
MIXED = [1, 780, 3, 0, 129], [70, 780, 900, 50, 1333]
WINDOWS = [(16, 0), (64, 1), (5, 33), (24, 128), (16, 1000)]
# few tokens over many places, which are cut, and many over few, which are not; window
LONG = [([80, 1], [5000, 777], 8, 1, 64, 32, 0), ([300], [2300], 4, 2, 128, 16, 0), ([2000], [2500], 2, 1, 256, 64, 1200), ([70], [9001], 3, 1, 256, 64, 0),
        ([1500] * 3, [1500, 2100, 1600], 8, 8, 64, 16, 0), ([900, 900], [1000, 1000], 8, 8, 128, 16, 800), ([300, 300], [400, 500], 4, 4, 256, 16, 0)]
# where values or keys are not finite
SPECIAL = [([470, 1], [500, 90], 16, 2, 128, 16, 0), ([470, 1], [500, 90], 16, 2, 128, 16, 25), ([1, 500], [100, 1400], 16, 2, 64, 16, 20),
           ([470], [470], 16, 2, 256, 16, 60), ([130], [2600], 4, 2, 128, 16, 0), ([40, 300], [1200, 2000], 4, 2, 80, 16, 1100)]
LARGE = [200], [264], 8, 1, 64, 16
NOTHING = [400, 300, 1, 200], [300, 0, 1, 700], 8, 2, 64, 16


def calls():
    """Every call of this file as tests/host_checks/attend_shape.cpp reads them."""
    def call(news, lengths, Hq, Hkv, D, page, width=None, window=0):
        return sum(news), len(news), Hq, Hkv, D, window, width or max(-(-n // page) for n in lengths), page
    out = [call(*c) for c in BEYOND_THE_TABLE]
    out += [call(*MIXED, *h, page, None, window) for h in HEADS for page, window in WINDOWS]
    out += [call(*c[:6], None, c[6]) for c in LONG + SPECIAL]
    out += [call(*LARGE), call(*NOTHING), call(*NOTHING, 19), call(*MIXED, 8, 1, 64, 16, None, 50), call(*MIXED, 6, 3, 64, 16), call(*MIXED, 8, 8, 128, 64)]
    return out


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("news,lengths,Hq,Hkv,D,page,width,window", BEYOND_THE_TABLE)
def test_lengths_beyond_the_table(ctx, dtype, news, lengths, Hq, Hkv, D, page, width, window):
    """Places that the table has no column for are attended to by nobody, wherever in a step of the kernel they begin."""
    a = inputs(dtype, news, lengths, Hq, Hkv, D, page)
    a["table"] = a["table"][:, :width]
    compare(ctx, a, dtype, window)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("page,window", WINDOWS)
def test_windows(ctx, dtype, Hq, Hkv, D, page, window):
    compare(ctx, inputs(dtype, *MIXED, Hq, Hkv, D, page), dtype, window)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("news,lengths,Hq,Hkv,D,page,window", LONG)
def test_pieces(ctx, dtype, news, lengths, Hq, Hkv, D, page, window):
    a = inputs(dtype, news, lengths, Hq, Hkv, D, page)
    got = compare(ctx, a, dtype, window)
    assert torch.equal(got, ctx.attend_pages(**a, window=window))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("special", [float("inf"), float("nan"), "lowest"])
@pytest.mark.parametrize("news,lengths,Hq,Hkv,D,page,window", SPECIAL)
def test_masked_places_have_no_part(ctx, dtype, special, news, lengths, Hq, Hkv, D, page, window):
    """Values and keys that are not finite reach the tokens that attend to them only."""
    special = torch.finfo(dtype).min if special == "lowest" else special
    a = inputs(dtype, news, lengths, Hq, Hkv, D, page)
    for r, (n, length) in enumerate(zip(news, lengths)):
        for u in {length - 1, length - n // 2 - 1, max(0, length - n - 21)}:
            at = int(a["table"][r, u // page])
            a["v_pages"][at, u % page, :, 3::5] = special
            a["k_pages"][at, u % page, 1] = special
    want, bound = F.attend(**a, window=window)
    got = ctx.attend_pages(**a, window=window).double().cpu()
    # where a token attends to them the definition is not finite, or too wide a sum for a bound: those are the others
    fine = (torch.isfinite(want) & (bound <= 1e3)).flatten()
    assert fine.any() and not fine.all()
    off = (got - want).abs().flatten()[fine]
    assert bool((off <= (bound + F.UNIT[dtype] * want.abs() + F.TINY[dtype]).flatten()[fine]).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("window", [0, 50])
def test_peaked_and_flat_weights(ctx, dtype, window):
    for spread in (30.0, 0.0):
        compare(ctx, inputs(dtype, *MIXED, 8, 1, 64, 16, spread=spread), dtype, window, spread)
    a = inputs(dtype, *MIXED, 8, 1, 64, 16)
    for scale in (0.0, -0.2):
        compare(ctx, dict(a, scale=scale), dtype, window, scale)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_rows_that_attend_to_nothing(ctx, dtype):
    """Lengths short of the new tokens, lengths of zero and less, pages that are not there."""
    a = inputs(dtype, *NOTHING)
    a["lengths"] = torch.tensor([300, -6, 1, 700], dtype=torch.int32, device="cuda")
    got = compare(ctx, a, dtype)
    assert not got[:100].any() and got[100:400].any(-1).all() and not got[400:700].any() and got[700:].any(-1).all()
    ctx.clear_bad_ids()
    a["table"][3, 1], a["table"][3, 20], a["table"][0, 0] = 1 << 20, -1, -2
    got = compare(ctx, a, dtype)
    assert not got[100:116].any() and got[116:400].any(-1).all() and got[700:].any(-1).all() and ctx.clear_bad_ids() > 0
    a["table"] = a["table"][:, :19]
    compare(ctx, a, dtype)
    # starts and lengths that are not what they should be: nothing outside the arrays is touched
    a["starts"] = torch.tensor([0, 1 << 30, -7, 300, 901], dtype=torch.int32, device="cuda")
    a["lengths"] = torch.tensor([1 << 30, 2 ** 31 - 1, -2 ** 31, 700], dtype=torch.int32, device="cuda")
    ctx.attend_pages(**a)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_other_orders_of_the_cache(ctx, dtype):
    """Heads before places, keys and values of a page side by side, queries and results as views of wider arrays."""
    a = inputs(dtype, *MIXED, 6, 3, 64, 16)
    want = compare(ctx, a, dtype)
    for turn in ((0, 2, 1, 3), (2, 0, 1, 3)):
        back = [turn.index(i) for i in range(4)]
        b = dict(a, k_pages=a["k_pages"].permute(turn).contiguous().permute(back), v_pages=a["v_pages"].permute(turn).contiguous().permute(back))
        assert torch.equal(ctx.attend_pages(**b), want)
    both = torch.stack([a["k_pages"], a["v_pages"]], 1)
    T = want.shape[0]
    row = torch.zeros(T, 12 * 64, dtype=dtype, device="cuda")
    q = row[:, 64:7 * 64].unflatten(1, (6, 64))
    q.copy_(a["q"])
    out = torch.zeros(T, 6, 128, dtype=dtype, device="cuda")
    got = ctx.attend_pages(**dict(a, k_pages=both[:, 0], v_pages=both[:, 1], q=q), out=out[:, :, 64:])
    assert torch.equal(got, want) and not out[:, :, :64].any()


def test_a_cache_beyond_four_giga_elements(ctx):
    """Places whose offsets pass 32 bits."""
    page, Hkv, D = 64, 8, 128
    pages = (1 << 32) // (page * Hkv * D) + 40
    k = torch.empty(pages, page, Hkv, D, dtype=BF16, device="cuda")
    v = torch.empty_like(k)
    a = inputs(BF16, *MIXED, 8, 8, D, page)
    where = torch.arange(a["k_pages"].shape[0], device="cuda")
    far = torch.where(where % 2 == 0, pages - 1 - where, where)
    k[far], v[far] = a["k_pages"], a["v_pages"]
    b = dict(a, k_pages=k, v_pages=v, table=torch.where(a["table"] >= 0, far[a["table"].clamp(min=0).long()], -1).int())
    assert torch.equal(ctx.attend_pages(**b), compare(ctx, a, BF16))


def test_values_near_the_largest_of_bf16(ctx):
    """Weighted sums that 32 bits hold if no weight is more than 1: values of 2^120, scores that rise by 6.9 bits once a row is under way."""
    a = inputs(BF16, *LARGE)
    a["q"].zero_()
    a["q"][..., 0] = 1
    a["k_pages"].zero_()
    a["v_pages"].copy_(torch.where(a["v_pages"].isnan(), a["v_pages"], a["v_pages"].sign() * 2.0 ** 120))
    for page in a["table"][0, 4:17]:
        a["k_pages"][int(page), :, :, 0] = 4.8
    compare(ctx, dict(a, scale=1.0), BF16)
