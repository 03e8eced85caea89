"""Places in a paged cache on the GPU against their definition, place by place (include/she_clear.h)."""
import random

import pytest
import torch

import clear_step_forms as F
import paper_1906_00148_amd as she

pytestmark = pytest.mark.gpu
I32 = torch.int32


@pytest.fixture(scope="module")
def ctx():
    with she.Context(she.TOY, 22, 64) as c:
        yield c


def dev(values, dtype=I32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def inputs(cached, news, page, width, seed=0, spare=0, extra=9, taken=3):
    """Pages in no order; columns that no request has hold -5."""
    rng = random.Random(seed)
    have = [-(-max(c, 0) // page) for c in cached]
    need = [-(-(max(c, 0) + max(n, 0)) // page) for c, n in zip(cached, news)]
    ids = list(range(sum(have) + taken + sum(need) + extra))
    rng.shuffle(ids)
    table = [[ids.pop() if column < h else -5 for column in range(width)] for h in have]
    pages = sum(have) + taken + sum(need) + extra
    return dict(cached=cached, news=news, table=table, free=ids, taken=taken, tokens=sum(max(n, 0) for n in news) + spare, pages=pages, page_size=page)


def compare(ctx, a, before=None, in_place=False):
    want = F.plan(**a, before=before)
    on = {k: dev(v) if isinstance(v, list) else v for k, v in a.items()}
    on["table"] = dev(a["table"]).reshape(len(a["cached"]), -1)
    on["taken"] = dev([a["taken"]])
    ctx.clear_bad_ids()
    out = None
    if in_place:
        R, T = len(a["cached"]), a["tokens"]
        out = (torch.empty(R + 1, dtype=I32, device="cuda"), on["cached"], torch.empty(T, dtype=I32, device="cuda"),
               torch.empty(T, dtype=torch.int64, device="cuda"), on["taken"])
    got = ctx.plan_pages(**on, before=None if before is None else dev(before), out=out)
    names = ("starts", "lengths", "positions", "slots", "taken")
    for name, g, w in zip(names, got, want):
        assert g.tolist() == ([w] if name == "taken" else w), name
    assert [t.dtype for t in got] == [I32, I32, I32, torch.int64, I32]
    assert on["table"].tolist() == want[5]
    assert ctx.clear_bad_ids() == want[6]
    if in_place:
        assert all(g is o for g, o in zip(got, out))
    return got, want


@pytest.mark.parametrize("page", [1, 2, 16, 24, 128])
@pytest.mark.parametrize("in_place", [False, True])
def test_small_steps(ctx, page, in_place):
    for cached, news in (([0], [1]), ([197], [1]), ([15, 16, 17, 0, 31, 32], [1] * 6), ([0, 0, 0], [0, 0, 0]), ([5, 0, 40], [0, 33, 17]),
                         ([127, 128, 129], [129, 1, 0]), ([0, 3], [1, 0])):
        a = inputs(cached, news, page, 320 // page + 2)
        compare(ctx, a, in_place=in_place)
        compare(ctx, dict(a, tokens=a["tokens"] + 5), before=[100 + r for r in range(len(cached))], in_place=in_place)


@pytest.mark.parametrize("requests,new", [(1, 5000), (63, 3), (64, 130), (500, 1), (4096, 1), (4097, 1), (4100, 2), (9000, 1)])
@pytest.mark.parametrize("in_place", [False, True])
def test_ragged_steps(ctx, requests, new, in_place):
    rng = random.Random(requests)
    cached = [rng.choice([0, rng.randint(0, 200)]) for _ in range(requests)]
    news = [new if requests == 1 else rng.choice([0, 1, rng.randint(0, new)]) for _ in range(requests)]
    a = inputs(cached, news, 16, (200 + new) // 16 + 1, spare=7)
    compare(ctx, a, before=[rng.randint(0, 99) for _ in range(requests)], in_place=in_place)


def test_long_runs_of_requests_that_pause(ctx):
    for requests in (300, 6000):
        news = [0] * requests
        news[7], news[200], news[requests - 1] = 3, 4200, 5
        compare(ctx, inputs([20] * requests, news, 16, 270))
        compare(ctx, inputs([20] * requests, [0] * (requests - 1) + [4500], 16, 300))


def test_room_for_fewer_tokens_than_there_are(ctx):
    for tokens in (0, 1, 16, 33, 34, 5000):
        compare(ctx, dict(inputs([0, 15, 31], [10, 20, 5], 16, 4), tokens=tokens))
        compare(ctx, dict(inputs([0, 15, 31], [10, 4990, 50], 16, 320), tokens=tokens))


@pytest.mark.parametrize("many", [False, True])
def test_pages_that_are_not_there(ctx, many):
    """A list that ends, ids out of range in it and in the table, tables short of columns: such tokens have no slot, and are counted."""
    n = 4200 if many else 40
    a = inputs([10, 16, 0, 33], [7, 1, n, 2], 16, n // 16 + 4)
    compare(ctx, dict(a, free=a["free"][:4]))
    compare(ctx, dict(a, free=a["free"][:3]))
    compare(ctx, dict(a, free=[]))
    compare(ctx, dict(a, taken=len(a["free"]) + 5))
    compare(ctx, dict(a, taken=-5))
    compare(ctx, dict(a, pages=a["pages"] // 2))
    compare(ctx, dict(a, pages=0))
    bad = [list(row) for row in a["table"]]
    bad[0][0], bad[3][2] = -7, 1 << 30
    compare(ctx, dict(a, table=bad))
    for width in (0, 1, 2, 3):
        compare(ctx, dict(a, table=[row[:width] for row in a["table"]]))


@pytest.mark.parametrize("many", [False, True])
def test_numbers_out_of_range(ctx, many):
    n = 4200 if many else 20
    a = inputs([-4, 5, 30], [3, -9, n], 16, n // 16 + 4)
    compare(ctx, a, before=[-3, 4, 2 ** 31 - 1])
    a = inputs([3, 7], [2, n], 16, n // 16 + 4)
    a["cached"] = [2 ** 31 - 2, 7]
    compare(ctx, a)
    a["news"] = [2 ** 31 - 1, 2 ** 31 - 1]
    compare(ctx, dict(a, cached=[3, 2 ** 31 - 1]))


def test_rows_of_a_wider_table(ctx):
    a = inputs([3, 40], [20, 9], 16, 4)
    wide = torch.full((2, 9), -8, dtype=I32, device="cuda")
    wide[:, 2:6] = dev(a["table"])
    want = F.plan(**a)
    on = {k: dev(v) if isinstance(v, list) else v for k, v in a.items()}
    got = ctx.plan_pages(**dict(on, table=wide[:, 2:6], taken=dev([a["taken"]])))
    assert got[3].tolist() == want[3] and wide[:, 2:6].tolist() == want[5]
    assert bool((wide[:, :2] == -8).all()) and bool((wide[:, 6:] == -8).all())


def test_no_requests(ctx):
    none = torch.zeros(0, dtype=I32, device="cuda")
    for tokens in (0, 3, 5000):
        got = ctx.plan_pages(none, none, none.view(0, 4), dev([1, 2]), dev([1]), tokens, 8, 16)
        assert got[0].tolist() == [0] and got[1].tolist() == [] and got[2].tolist() == [0] * tokens and got[3].tolist() == [-1] * tokens and got[4].tolist() == [1]


@pytest.mark.parametrize("requests", [5, 5000])
def test_steps_in_a_graph_go_on_from_one_another(ctx, requests):
    """Lengths and the list's entry in place: every replay is a step more."""
    a = inputs([3] * requests, [1] * requests, 4, 8, extra=9 * requests)
    on = {k: dev(v) if isinstance(v, list) else v for k, v in a.items()}
    on["taken"] = dev([a["taken"]])
    out = (torch.empty(requests + 1, dtype=I32, device="cuda"), on["cached"], torch.empty(requests, dtype=I32, device="cuda"),
           torch.empty(requests, dtype=torch.int64, device="cuda"), on["taken"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ctx.set_stream(side.cuda_stream)
    state = dict(a)

    def check():
        want = F.plan(**state)
        assert [g.tolist() for g in out] == [want[0], want[1], want[2], want[3], [want[4]]] and on["table"].tolist() == want[5]
        state.update(cached=want[1], taken=want[4], table=want[5])
    try:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            ctx.plan_pages(**on, out=out)
            side.synchronize()
            check()
            with torch.cuda.graph(graph, stream=side):
                ctx.plan_pages(**on, out=out)
        for _ in range(6):
            graph.replay()
            torch.cuda.synchronize()
            check()
    finally:
        ctx.set_stream(0)


def test_refusals(ctx):
    a = inputs([3, 40], [20, 9], 16, 4)
    on = {k: dev(v) if isinstance(v, list) else v for k, v in a.items()}
    on["taken"] = dev([a["taken"]])
    for bad in (dict(cached=on["cached"][:1]), dict(news=on["news"].long()), dict(table=on["table"].cpu()), dict(table=on["table"].mT), dict(free=on["free"].float()),
                dict(taken=dev([1, 2])), dict(taken=None), dict(cached=None), dict(tokens=-1), dict(tokens=(1 << 24) + 1), dict(pages=-1), dict(page_size=0),
                dict(page_size=1 << 26), dict(before=dev([1])), dict(news=dev([1, 2, 3]))):
        with pytest.raises(she.SheError):
            ctx.plan_pages(**{**on, **bad})
