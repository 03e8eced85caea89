"""Attention over a paged cache on the GPU against its definition in 64 bits (include/she_clear.h)."""
import pytest
import torch

import clear_forms as F
import paper_1906_00148_amd as she

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    with she.Context(she.TOY, 13, 64) as c:
        yield c


def inputs(dtype, news, lengths, Hq, Hkv, D, page, seed=0, spread=1.0):
    """Pages whose slots beyond a request's length, and spare pages, hold NaN."""
    g = torch.Generator().manual_seed(seed)
    table, pages = F.pages_of([max(n, 0) for n in lengths], page, seed=seed)
    kv = torch.full((2, pages, page, Hkv, D), float("nan"))
    for r, n in enumerate(lengths):
        for u in range(0, n, page):
            m = min(page, n - u)
            kv[:, table[r, u // page], :m] = torch.randn(2, m, Hkv, D, generator=g)
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    k, v = kv.to(dtype).cuda()
    return dict(q=(torch.randn(starts[-1], Hq, D, generator=g) * spread).to(dtype).cuda(), k_pages=k, v_pages=v, table=table.cuda(),
                starts=torch.tensor(starts, dtype=torch.int32).cuda(), lengths=torch.tensor(lengths, dtype=torch.int32).cuda(), scale=D ** -0.5)


def compare(ctx, a, dtype, window=0, what=""):
    got = ctx.attend_pages(**a, window=window)
    want, bound = F.attend(**a, window=window)
    F.check(got, want, bound, dtype, what)
    return got


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (4, 4, 128), (8, 1, 80), (7, 1, 96), (6, 2, 256), (3, 1, 192), (2, 2, 8), (5, 5, 40)])
@pytest.mark.parametrize("page", [16, 1, 24])
def test_single_tokens(ctx, dtype, Hq, Hkv, D, page):
    lengths = [1, 2, 31, 32, 33, 64, 129, 300, 257]
    compare(ctx, inputs(dtype, [1] * len(lengths), lengths, Hq, Hkv, D, page), dtype)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (4, 4, 128), (7, 1, 96), (6, 2, 256)])
@pytest.mark.parametrize("page,window", [(16, 0), (64, 0), (5, 0), (16, 1), (64, 33), (16, 100)])
def test_chunks_and_tokens_together(ctx, dtype, Hq, Hkv, D, page, window):
    compare(ctx, inputs(dtype, [1, 40, 3, 129, 0, 17], [70, 40, 200, 190, 50, 17], Hq, Hkv, D, page), dtype, window)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("news,lengths", [([300], [300]), ([257], [900]), ([1], [5000]), ([2], [4097]), ([65, 1], [2500, 3000])])
def test_long_caches_that_workgroups_share(ctx, dtype, news, lengths):
    a = inputs(dtype, news, lengths, 4, 1, 128, 32)
    got = compare(ctx, a, dtype)
    assert torch.equal(got, ctx.attend_pages(**a))


@pytest.mark.parametrize("Hq,Hkv", [(16, 1), (17, 1), (40, 2), (33, 1)])
@pytest.mark.parametrize("news", [[1], [9], [1, 1, 1], [1, 0, 5, 1], [2, 30, 1]])
def test_many_query_heads_for_a_key_head(ctx, Hq, Hkv, news):
    """A token alone has more rows than a tile of the kernel for few rows, or just as many."""
    a = inputs(BF16, news, [700 + 60 * i for i in range(len(news))], Hq, Hkv, 64, 16)
    for window in (0, 90):
        compare(ctx, a, BF16, window)


@pytest.mark.parametrize("window", [0, 50])
def test_peaked_and_flat_weights(ctx, window):
    for spread in (30.0, 0.0):
        compare(ctx, inputs(F16, [1, 70], [400, 230], 4, 2, 64, 16, spread=spread), F16, window, spread)
    a = inputs(BF16, [1, 70], [400, 230], 4, 2, 64, 16)
    a["scale"] = 0.0
    compare(ctx, a, BF16, window)
    a["scale"] = -0.2
    compare(ctx, a, BF16, window)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("special", [float("inf"), float("nan"), "lowest"])
def test_masked_places_have_no_part(ctx, dtype, special):
    """Values and keys of later tokens and of places before the window that are not finite reach the tokens that attend to them only."""
    special = torch.finfo(dtype).min if special == "lowest" else special
    for news, lengths, window in (([40], [100], 0), ([40], [100], 25), ([1, 30, 150], [90, 30, 400], 20), ([3], [3], 0), ([9], [500], 60)):
        a = inputs(dtype, news, lengths, 4, 2, 128, 16)
        size = 16
        for r, (n, length) in enumerate(zip(news, lengths)):
            for u in {length - 1, length - n // 2 - 1, max(0, length - 70), max(0, length - 21)}:
                page = int(a["table"][r, u // size])
                a["v_pages"][page, u % size, :, 3::5] = special
                a["k_pages"][page, u % size, 1] = special
        want, bound = F.attend(**a, window=window)
        got = ctx.attend_pages(**a, window=window).double().cpu()
        fine = torch.isfinite(want)
        assert fine.any()
        # where a token attends to them the definition is not finite, or too wide a sum for a bound: those are the others
        wide = bound > 1e3
        assert bool(torch.isfinite(got)[fine & ~wide].all()), (news, lengths, window)
        ok = (fine & ~wide).flatten()
        off = (got - want).abs().flatten()[ok]
        assert bool((off <= (bound + F.UNIT[dtype] * want.abs() + F.TINY[dtype]).flatten()[ok]).all())


def test_rows_that_attend_to_nothing(ctx):
    """Lengths short of the new tokens, lengths of zero, tables without a column, pages that are not there."""
    a = inputs(BF16, [5, 3, 1, 2], [3, 0, 1, 40], 4, 2, 64, 16)
    a["lengths"] = torch.tensor([3, 0, -6, 40], dtype=torch.int32, device="cuda")
    got = compare(ctx, a, BF16)
    assert not got[:2].any() and not got[5:9].any() and got[2].any() and got[9:].any()
    ctx.clear_bad_ids()
    a["table"][3, 1], a["table"][0, 0] = 1 << 20, -2
    got = compare(ctx, a, BF16)
    assert not got[:5].any() and got[9:].any() and ctx.clear_bad_ids() > 0
    a["table"] = a["table"][:, :1]
    compare(ctx, a, BF16)
    a["table"] = a["table"][:, :0]
    assert not ctx.attend_pages(**a).any()
    a = inputs(BF16, [0, 0], [20, 3], 4, 2, 64, 16)
    assert ctx.attend_pages(**a).shape == (0, 4, 64)
    # starts and lengths that are not what they should be: nothing outside the arrays is touched
    a = inputs(BF16, [20, 30], [20, 64], 4, 2, 64, 16)
    a["starts"] = torch.tensor([0, 1 << 30, -7], dtype=torch.int32, device="cuda")
    a["lengths"] = torch.tensor([1 << 30, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    ctx.attend_pages(**a)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_other_orders_of_the_cache(ctx, dtype):
    """Heads before places, keys and values of a page side by side, queries as views of one projection."""
    a = inputs(dtype, [1, 30], [100, 77], 6, 3, 64, 16)
    want = ctx.attend_pages(**a)
    for turn in ((0, 2, 1, 3), (2, 0, 1, 3)):
        back = [turn.index(i) for i in range(4)]
        b = dict(a, k_pages=a["k_pages"].permute(turn).contiguous().permute(back), v_pages=a["v_pages"].permute(turn).contiguous().permute(back))
        assert torch.equal(ctx.attend_pages(**b), want)
    both = torch.stack([a["k_pages"], a["v_pages"]], 1)
    row = torch.zeros(31, 12 * 64, dtype=dtype, device="cuda")
    q = row[:, 64:7 * 64].unflatten(1, (6, 64))
    q.copy_(a["q"])
    out = torch.zeros(31, 6, 128, dtype=dtype, device="cuda")
    got = ctx.attend_pages(**dict(a, k_pages=both[:, 0], v_pages=both[:, 1], q=q), out=out[:, :, 64:])
    assert torch.equal(got, want) and not out[:, :, :64].any()
    wide = torch.full((2, 40), -1, dtype=torch.int32, device="cuda")
    wide[:, :a["table"].shape[1]] = a["table"]
    assert torch.equal(ctx.attend_pages(**dict(a, table=wide[:, :a["table"].shape[1]])), want)


def test_a_cache_beyond_four_giga_elements(ctx):
    """Places whose offsets pass 32 bits."""
    page, Hkv, D = 64, 8, 128
    pages = (1 << 32) // (page * Hkv * D) + 8
    k = torch.empty(pages, page, Hkv, D, dtype=BF16, device="cuda")
    v = torch.empty_like(k)
    a = inputs(BF16, [1, 33], [150, 190], 8, 8, D, page)
    where = torch.arange(a["k_pages"].shape[0], device="cuda")
    far = torch.where(where % 2 == 0, pages - 1 - where, where)
    k[far], v[far] = a["k_pages"], a["v_pages"]
    b = dict(a, k_pages=k, v_pages=v, table=torch.where(a["table"] >= 0, far[a["table"].clamp(min=0).long()], -1).int())
    assert torch.equal(ctx.attend_pages(**b), ctx.attend_pages(**a))


def test_on_another_stream_and_in_a_graph(ctx):
    a = inputs(BF16, [1, 200, 1], [3000, 600, 80], 8, 2, 128, 16)
    want = ctx.attend_pages(**a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a["q"] = a["q"] + 0
        got = ctx.attend_pages(**a)
        total = got.float().sum()
    side.synchronize()
    assert torch.equal(got, want) and torch.isfinite(total)
    with torch.cuda.graph(torch.cuda.CUDAGraph()):                # the context's stream is the default one: it cannot be captured
        with pytest.raises(she.SheError):
            ctx.attend_pages(**a)
    ctx.set_stream(side.cuda_stream)
    try:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = ctx.attend_pages(**a)
        for k in range(3):
            a["q"].copy_(torch.randn_like(a["q"]))
            want = ctx.attend_pages(**a)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, want), k
    finally:
        ctx.set_stream(0)


def test_refusals(ctx):
    a = inputs(BF16, [1, 2], [20, 30], 4, 2, 64, 16)

    def refused(code, **changed):
        with pytest.raises(she.SheError) as e:
            ctx.attend_pages(**dict(a, **changed))
        assert e.value.code == code, e.value
    refused(-1, q=a["q"].float())
    refused(-1, q=a["q"][:, :3])
    refused(-1, q=a["q"][..., :60], k_pages=a["k_pages"][..., :60], v_pages=a["v_pages"][..., :60])
    refused(-1, k_pages=a["k_pages"].half())
    refused(-1, v_pages=a["v_pages"][:, :8])
    refused(-1, table=a["table"].long())
    refused(-1, starts=a["starts"][:2])
    refused(-1, lengths=a["lengths"].float())
    refused(-1, window=-1)
    refused(-1, out=torch.empty_like(a["q"])[:2])
    shifted = torch.zeros(3 * 4 * 64 + 1, dtype=BF16, device="cuda")[1:].view(3, 4, 64)
    refused(-1, q=shifted)
    huge = torch.zeros(1, 1, 2, 264, dtype=BF16, device="cuda")
    refused(-1, q=torch.zeros(3, 4, 264, dtype=BF16, device="cuda"), k_pages=huge, v_pages=huge)
    refused(-4, table=torch.zeros(2, (1 << 22) + 1, dtype=torch.int32, device="cuda"))


def test_a_capture_never_allocates_and_outlives_the_scratch_it_had():
    small, large = inputs(BF16, [1], [1500], 4, 1, 128, 16), inputs(BF16, [1, 1], [60000, 300], 8, 8, 128, 64)
    side = torch.cuda.Stream()
    with she.Context(she.TOY, 14, 64) as c:
        c.set_stream(side.cuda_stream)
        want = c.attend_pages(**small)                            # the cut rows' pieces need scratch
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            with pytest.raises(she.SheError) as e:
                c.attend_pages(**large)
            assert e.value.code == -2
            got = c.attend_pages(**small)
        c.attend_pages(**large)                                   # grows it
        torch.cuda.synchronize()
        junk = torch.randn(1 << 20, device="cuda")                # whatever is allocated next
        for _ in range(3):
            got.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, want) and bool(torch.isfinite(junk).all())
