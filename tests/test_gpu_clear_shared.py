"""Attention behind shared prefixes on the GPU against its definition in 64 bits (include/she_clear.h)."""
import pytest
import torch

import clear_forms as C
import clear_step_forms as F
import paper_1906_00148_amd as she

pytestmark = pytest.mark.gpu
BF16, F16, I32 = torch.bfloat16, torch.float16, torch.int32


@pytest.fixture(scope="module")
def ctx():
    with she.Context(she.TOY, 23, 64) as c:
        yield c


def inputs(dtype, groups, Hq, Hkv, D, page, before=(), after=(), seed=0, spread=1.0):
    """groups: for each prefix its length and its requests, (new tokens, own places) each; before, after: requests without a prefix.
    Slots of pages beyond a length, and spare pages, hold NaN."""
    g = torch.Generator().manual_seed(seed)
    requests = [*before, *(r for _, rs in groups for r in rs), *after]
    prefixes = [n for n, _ in groups]
    counts = [max(n, 0) for n in prefixes] + [max(n, 0) for _, n in requests]
    table, pages = C.pages_of(counts, page, seed=seed)
    kv = torch.full((2, pages, page, Hkv, D), float("nan"))
    for row, n in zip(table, counts):
        for u in range(0, n, page):
            m = min(page, n - u)
            kv[:, row[u // page], :m] = torch.randn(2, m, Hkv, D, generator=g)
    starts, ranges = [0], [len(before)]
    for n, _ in requests:
        starts.append(starts[-1] + n)
    for _, rs in groups:
        ranges.append(ranges[-1] + len(rs))
    k, v = kv.to(dtype).cuda()
    i32 = lambda x: torch.tensor(x, dtype=I32, device="cuda")
    G = len(groups)

    def narrow(rows, some):
        return table[rows][:, :max([-(-max(n, 0) // page) for n in some] + [1])].contiguous().cuda()
    return dict(q=(torch.randn(starts[-1], Hq, D, generator=g) * spread).to(dtype).cuda(), k_pages=k, v_pages=v,
                table=narrow(slice(G, None), [n for _, n in requests]), starts=i32(starts), lengths=i32([n for _, n in requests]),
                prefix_table=narrow(slice(0, G), prefixes), prefix_requests=i32(ranges), prefix_lengths=i32(prefixes), scale=D ** -0.5)


def compare(ctx, a, dtype, window=0, what=""):
    got = ctx.attend_shared(**a, window=window)
    want, bound = F.shared(**a, window=window)
    C.check(got, want, bound, dtype, what)
    return got


HEADS = [(8, 2, 64), (4, 4, 128), (8, 1, 80), (7, 1, 96), (6, 2, 256), (3, 1, 192), (2, 2, 8), (5, 5, 40)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("page", [16, 1, 24])
def test_tokens_behind_one_prefix(ctx, dtype, Hq, Hkv, D, page):
    compare(ctx, inputs(dtype, [(133, [(1, 1), (1, 20), (1, 33)])], Hq, Hkv, D, page), dtype)
    compare(ctx, inputs(dtype, [(300, [(1, n) for n in range(1, 41)])], Hq, Hkv, D, page), dtype)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (4, 4, 128), (7, 1, 96), (6, 2, 256)])
@pytest.mark.parametrize("page,window", [(16, 0), (64, 0), (5, 0), (16, 1), (64, 33), (16, 100), (16, 260)])
def test_several_prefixes_chunks_and_tokens(ctx, dtype, Hq, Hkv, D, page, window):
    groups = [(200, [(1, 30), (40, 41), (3, 90)]), (1, [(129, 129)]), (77, [(1, 1), (0, 5), (17, 50)]), (0, [(2, 9)]), (64, [])]
    compare(ctx, inputs(dtype, groups, Hq, Hkv, D, page, before=[(5, 9)], after=[(1, 44), (33, 70)]), dtype, window)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("requests,prefix", [(1, 5000), (2, 4097), (16, 2500), (33, 3000), (64, 2048), (130, 1500), (300, 700)])
@pytest.mark.parametrize("window", [0, 1024])
def test_long_prefixes_that_workgroups_share(ctx, dtype, requests, prefix, window):
    a = inputs(dtype, [(prefix, [(1, 1 + r % 7) for r in range(requests)])], 4, 1, 128, 32)
    got = compare(ctx, a, dtype, window)
    assert torch.equal(got, ctx.attend_shared(**a, window=window))


@pytest.mark.parametrize("Hkv", [1, 8])
def test_long_own_places(ctx, Hkv):
    """The requests' own places are cut too."""
    compare(ctx, inputs(BF16, [(700, [(1, 3000), (2, 2100)])], 2 * Hkv, Hkv, 64, 16), BF16)
    compare(ctx, inputs(BF16, [(40, [(150, 1500)])], 2 * Hkv, Hkv, 64, 16), BF16)


@pytest.mark.parametrize("Hq,Hkv", [(16, 1), (17, 1), (40, 2), (129, 1)])
def test_many_query_heads_for_a_key_head(ctx, Hq, Hkv):
    for window in (0, 90):
        compare(ctx, inputs(BF16, [(500, [(1, 3)]), (90, [(9, 20), (1, 2), (1, 60)])], Hq, Hkv, 64, 16), BF16, window)


@pytest.mark.parametrize("window", [0, 50])
def test_peaked_and_flat_weights(ctx, window):
    groups = [(400, [(1, 30), (70, 80)]), (230, [(1, 9)] * 20)]
    for spread in (30.0, 0.0):
        compare(ctx, inputs(F16, groups, 4, 2, 64, 16, spread=spread), F16, window, spread)
    for scale in (0.0, -0.2):
        compare(ctx, dict(inputs(BF16, groups, 4, 2, 64, 16), scale=scale), BF16, window)


@pytest.mark.parametrize("page", [16, 64])
def test_as_attention_over_both_in_one_row(ctx, page):
    """A prefix of whole pages and a request's own pages are one request of attend_pages."""
    a = inputs(BF16, [(8 * page, [(1, 40), (30, 30), (2, 70)]), (3 * page, [(1, 1), (5, 100)])], 8, 2, 128, page)
    width = a["table"].shape[1] + 8
    both = torch.full((5, width), -1, dtype=I32)
    lengths = []
    for r, (g, pages) in enumerate([(0, 8)] * 3 + [(1, 3)] * 2):
        both[r, :pages] = a["prefix_table"][g, :pages].cpu()
        both[r, pages:pages + a["table"].shape[1]] = a["table"][r].cpu()
        lengths.append(pages * page + a["lengths"][r].item())
    for window in (0, 3 * page):
        want = ctx.attend_pages(a["q"], a["k_pages"], a["v_pages"], both.cuda(), a["starts"], torch.tensor(lengths, dtype=I32, device="cuda"), window=window)
        got = ctx.attend_shared(**a, window=window)
        _, bound = F.shared(**a, window=window)
        assert bool(((got.double() - want.double()).abs().cpu() <= 2 * bound + 2 * C.UNIT[BF16] * want.double().abs().cpu()).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("special", [float("inf"), float("nan"), "lowest"])
@pytest.mark.parametrize("requests", [2, 40])
def test_masked_places_have_no_part(ctx, dtype, special, requests):
    """Keys and values that are not finite reach the tokens that attend to them only: before a window that begins in the prefix, and own
    places of later tokens."""
    special = torch.finfo(dtype).min if special == "lowest" else special
    page, window, prefix = 16, 60, 150
    a = inputs(dtype, [(prefix, [(1 + r % 3, 5 + (r * 7) % 50) for r in range(requests)]), (prefix, [(20, 30)])], 4, 2, 128, page)
    for g in (0, 1):
        for u in (0, 3, 95, 120, 149):
            at = int(a["prefix_table"][g, u // page])
            a["v_pages"][at, u % page, :, 3::5] = special
            a["k_pages"][at, u % page, 1] = special
    at = int(a["table"][requests, 29 // page])
    a["v_pages"][at, 29 % page, :, 3::5] = special
    for w in (window, 0, 20):
        want, bound = F.shared(**a, window=w)
        got = ctx.attend_shared(**a, window=w).double().cpu()
        fine, wide = torch.isfinite(want), bound > 1e3
        assert bool(torch.isfinite(got)[fine & ~wide].all()), w
        ok = (fine & ~wide).flatten()
        assert ok.any() or w == 0
        off = (got - want).abs().flatten()[ok]
        assert bool((off <= (bound + C.UNIT[dtype] * want.abs() + C.TINY[dtype]).flatten()[ok]).all())


@pytest.mark.parametrize("window", [0, 40])
def test_rows_that_attend_to_nothing(ctx, window):
    """Own lengths short of the new tokens, prefixes of no places, tables without a column, pages that are not there."""
    a = inputs(BF16, [(50, [(5, 3), (3, 0), (1, 1)]), (0, [(2, 40), (1, 0)])], 4, 2, 64, 16)
    a["lengths"] = torch.tensor([3, 0, -6, 40, 0], dtype=I32, device="cuda")
    got = compare(ctx, a, BF16, window)
    assert not got[:2].any() and got[2].any() and not got[5:9].any() and got[9:11].any() and not got[11].any()
    a["lengths"] = torch.tensor([5, 3, 1, 40, 1], dtype=I32, device="cuda")
    ctx.clear_bad_ids()
    compare(ctx, a, BF16, window)
    b = dict(a, table=a["table"].clone(), prefix_table=a["prefix_table"].clone())
    b["prefix_table"][0, 2], b["table"][3, 1] = -1, 1 << 20
    ctx.clear_bad_ids()
    compare(ctx, b, BF16, window)
    assert ctx.clear_bad_ids() > 0
    for rows in (dict(table=a["table"][:, :1]), dict(prefix_table=a["prefix_table"][:, :1]), dict(table=a["table"][:, :0]), dict(prefix_table=a["prefix_table"][:, :0])):
        compare(ctx, {**a, **rows}, BF16, window)
    b = dict(a, prefix_table=torch.full_like(a["prefix_table"], -1), table=torch.full_like(a["table"], 1 << 30))
    assert not ctx.attend_shared(**b, window=window).any()
    a["prefix_lengths"] = torch.tensor([-7, -2 ** 31], dtype=I32, device="cuda")
    compare(ctx, a, BF16, window)
    # numbers that are not what they should be: nothing outside the arrays is touched
    a["prefix_lengths"] = torch.tensor([2 ** 31 - 1, 1 << 30], dtype=I32, device="cuda")
    a["lengths"] = torch.tensor([1 << 30, 2 ** 31 - 1, -1, 7, 1], dtype=I32, device="cuda")
    ctx.attend_shared(**a, window=window)
    for ranges in ([-5, 9, 1 << 30], [4, 2, 0], [1 << 30, -1, 3]):
        ctx.attend_shared(**dict(a, prefix_requests=torch.tensor(ranges, dtype=I32, device="cuda")), window=window)
    ctx.attend_shared(**dict(a, starts=torch.tensor([0, 1 << 30, -7, 3, 100, 2], dtype=I32, device="cuda")), window=window)
    torch.cuda.synchronize()


def test_without_a_prefix_or_a_request(ctx):
    a = inputs(BF16, [], 4, 2, 64, 16, after=[(1, 20), (7, 30)])
    a["prefix_requests"] = torch.zeros(1, dtype=I32, device="cuda")
    got = compare(ctx, a, BF16)
    want = ctx.attend_pages(*(a[k] for k in ("q", "k_pages", "v_pages", "table", "starts", "lengths")))
    assert bool(((got.double() - want.double()).abs() <= 2 * C.UNIT[BF16] * (want.double().abs() + 1)).all())
    a = inputs(BF16, [(30, [(0, 20), (0, 3)])], 4, 2, 64, 16)
    assert ctx.attend_shared(**a).shape == (0, 4, 64)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("tokens", [1, 60])
def test_other_orders_of_the_cache(ctx, dtype, tokens):
    """Heads before places, keys and values of a page side by side, queries and results as views of wider rows."""
    a = inputs(dtype, [(100, [(tokens, tokens + 10), (1, 77)]), (40, [(1, 5)])], 6, 3, 64, 16)
    T = tokens + 2
    want = ctx.attend_shared(**a)
    for turn in ((0, 2, 1, 3), (2, 0, 1, 3)):
        back = [turn.index(i) for i in range(4)]
        b = dict(a, k_pages=a["k_pages"].permute(turn).contiguous().permute(back), v_pages=a["v_pages"].permute(turn).contiguous().permute(back))
        assert torch.equal(ctx.attend_shared(**b), want)
    both = torch.stack([a["k_pages"], a["v_pages"]], 1)
    q = torch.zeros(T, 12 * 64, dtype=dtype, device="cuda")[:, 64:7 * 64].unflatten(1, (6, 64))
    q.copy_(a["q"])
    out = torch.full((T + 3, 6, 128), 7.0, dtype=dtype, device="cuda")
    got = ctx.attend_shared(**dict(a, k_pages=both[:, 0], v_pages=both[:, 1], q=q), out=out[:T, :, 64:])
    assert torch.equal(got, want) and bool((out[:, :, :64] == 7).all()) and bool((out[T:] == 7).all())


def test_tokens_behind_the_last_request_are_left_as_they_were(ctx):
    a = inputs(BF16, [(60, [(1, 5), (2, 9)])], 4, 2, 64, 16)
    q = torch.cat([a["q"], torch.full((4, 4, 64), float("nan"), dtype=BF16, device="cuda")])
    out = torch.full((7, 4, 64), 3.0, dtype=BF16, device="cuda")
    ctx.attend_shared(**dict(a, q=q), out=out)
    assert torch.equal(out[:3], ctx.attend_shared(**a)) and bool((out[3:] == 3).all())


def test_on_another_stream_and_in_a_graph(ctx):
    a = inputs(BF16, [(500, [(1, 5 + r) for r in range(20)]), (90, [(4, 9)])], 8, 2, 128, 16)
    want = ctx.attend_shared(**a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ctx.attend_shared(**a)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    ctx.set_stream(side.cuda_stream)
    try:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            ctx.attend_shared(**a)
            side.synchronize()
            with torch.cuda.graph(graph, stream=side):
                out = ctx.attend_shared(**a)
    finally:
        ctx.set_stream(0)
    for seed in (None, 3, 4):
        if seed:
            a["q"].copy_(torch.randn(a["q"].shape, generator=torch.Generator().manual_seed(seed)))
            a["prefix_lengths"][0] = 500 - 100 * seed
            want = ctx.attend_shared(**a)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_refusals(ctx):
    a = inputs(BF16, [(50, [(1, 3), (2, 9)])], 4, 2, 64, 16)
    for bad in (dict(q=a["q"].float()), dict(q=a["q"].cpu()), dict(k_pages=a["k_pages"].half()), dict(k_pages=a["k_pages"][:, :, :, :40]), dict(starts=a["starts"][:2]),
                dict(lengths=a["lengths"].long()), dict(prefix_table=a["prefix_table"].mT), dict(prefix_requests=a["prefix_lengths"]),
                dict(prefix_lengths=a["lengths"]), dict(prefix_lengths=a["prefix_lengths"].float()), dict(prefix_requests=None), dict(table=a["table"].cpu()),
                dict(window=-1), dict(window=1 << 32), dict(out=a["q"].float()), dict(q=a["q"][:, :3])):
        with pytest.raises(she.SheError):
            ctx.attend_shared(**{**a, **bad})


def test_gradients_are_not_lost_in_silence(ctx):
    a = inputs(BF16, [(50, [(1, 3), (2, 9)])], 4, 2, 64, 16)
    for name in ("q", "k_pages", "v_pages"):
        out = ctx.attend_shared(**dict(a, **{name: a[name].clone().requires_grad_()}))
        with pytest.raises(she.SheError):
            out.float().sum().backward()
