"""Steps of generation with the calls as they are used together: places in the cache, keys and values into it, attention behind a shared
prefix, the next token; every step against the definitions in 64 bits, eager and captured (include/she_clear.h)."""
import pytest
import torch

import clear_forms as C
import clear_step_forms as F
import paper_1906_00148_amd as she

pytestmark = pytest.mark.gpu
I32 = torch.int32
HQ, HKV, D, PAGE, PAGES, WIDTH, VOCAB, POSITIONS = 8, 2, 64, 16, 64, 5, 9001, 256
EPS = 1e-6


@pytest.fixture(scope="module")
def ctx():
    with she.Context(she.TOY, 29, 64) as c:
        yield c


def dev(values, dtype=I32):
    return torch.tensor(values, dtype=dtype, device="cuda")


class Session:
    """Two texts that requests begin with, and requests behind them: one block of attention between an embedding and logits."""

    def __init__(self, ctx, dtype, texts, groups, room, seed=0):
        g = torch.Generator().manual_seed(seed)
        R = sum(groups)
        self.ctx, self.dtype, self.R, self.room = ctx, dtype, R, room
        self.embedding = torch.randn(VOCAB, (HQ + 2 * HKV) * D, generator=g).to(dtype).cuda()
        self.head = (torch.randn(HQ * D, VOCAB, generator=g) / 4).to(dtype).cuda()
        self.wq, self.wk = (1 + 0.1 * torch.randn(2, D, generator=g)).cuda()
        angle = torch.arange(POSITIONS)[:, None] * 100.0 ** (-torch.arange(D // 2) * 2.0 / D)
        self.cos, self.sin = angle.cos().cuda(), angle.sin().cuda()
        self.k_pages, self.v_pages = torch.full((2, PAGES, PAGE, HKV, D), float("nan"), dtype=dtype, device="cuda")
        self.free = torch.randperm(PAGES, generator=g).to(I32).cuda()
        self.taken = dev([0])
        self.table = torch.full((R, WIDTH), -1, dtype=I32, device="cuda")
        self.lengths = torch.zeros(R, dtype=I32, device="cuda")
        self.uniform = torch.zeros(R, device="cuda")
        self.temperature = torch.linspace(0, 1.5, R, device="cuda")
        self.top_k, self.top_p = dev([(0, 50)[r % 2] for r in range(R)]), torch.linspace(0.6, 1, R, device="cuda")
        # the texts are requests of a step of their own, whose table and lengths are the prefixes' from then on
        self.prefix_table = torch.full((len(texts), WIDTH), -1, dtype=I32, device="cuda")
        ids = torch.randint(0, VOCAB, (sum(texts),), generator=g).cuda()
        starts, self.prefix_lengths, positions, slots, self.taken = ctx.plan_pages(
            torch.zeros_like(dev(texts)), dev(texts), self.prefix_table, self.free, self.taken, sum(texts), PAGES, PAGE)
        self.turn(ids, positions, slots)
        ranges = [0]
        for n in groups:
            ranges.append(ranges[-1] + n)
        self.prefix_requests = dev(ranges)
        self.before = torch.cat([self.prefix_lengths[i].expand(n) for i, n in enumerate(groups)]).contiguous()

    def turn(self, ids, positions, slots):
        q, k, v = (t.unflatten(1, (-1, D)) for t in self.embedding[ids].split([HQ * D, HKV * D, HKV * D], 1))
        return (q, k, v), self.ctx.qk_rotate_append(q, k, v, self.wq, self.wk, self.cos, self.sin, positions, self.k_pages, self.v_pages, slots, eps=EPS)

    def step(self, ids, news):
        """`ids` [room]: the requests' new tokens one behind another; returns all that comes up on the way."""
        ctx = self.ctx
        starts, _, positions, slots, _ = plan = ctx.plan_pages(
            self.lengths, news, self.table, self.free, self.taken, self.room, PAGES, PAGE, before=self.before,
            out=(torch.empty(self.R + 1, dtype=I32, device="cuda"), self.lengths, torch.empty(self.room, dtype=I32, device="cuda"),
                 torch.empty(self.room, dtype=torch.int64, device="cuda"), self.taken))
        heads, turned = self.turn(ids, positions, slots)
        attended = torch.zeros_like(turned)
        ctx.attend_shared(turned, self.k_pages, self.v_pages, self.table, starts, self.lengths, self.prefix_table, self.prefix_requests,
                          self.prefix_lengths, out=attended)
        logits = attended[(starts[1:] - 1).long()].flatten(1) @ self.head
        chosen = ctx.sample(logits, self.uniform, temperature=self.temperature, top_k=self.top_k, top_p=self.top_p)
        return dict(plan=plan, heads=heads, turned=turned, attended=attended, logits=logits, chosen=chosen)

    def host(self):
        return dict(cached=self.lengths.tolist(), table=self.table.tolist(), taken=int(self.taken), k=self.k_pages.clone(), v=self.v_pages.clone())

    def check(self, was, news, got):
        starts, lengths, positions, slots, taken, table, lost = F.plan(was["cached"], news, was["table"], self.free.tolist(), was["taken"], self.room, PAGES, PAGE,
                                                                       self.before.tolist())
        assert [t.tolist() for t in got["plan"]] == [starts, lengths, positions, slots, [taken]] and self.table.tolist() == table and lost == 0
        (q, k, v), live, dtype = got["heads"], starts[-1], self.dtype
        at = torch.tensor(positions)
        C.check(got["turned"], *C.rotate(q, self.wq, self.cos, self.sin, at, EPS, False), dtype)
        k_now, v_now = (t.flatten(0, 1) for t in (self.k_pages, self.v_pages))
        new = torch.tensor(slots[:live])
        C.check(k_now[new.cuda()], *C.rotate(k[:live], self.wk, self.cos, self.sin, at[:live], EPS, False), dtype)
        assert torch.equal(v_now[new.cuda()], v[:live])
        others = torch.ones(PAGES * PAGE, dtype=torch.bool)
        others[new] = False
        for now, before in ((k_now, was["k"]), (v_now, was["v"])):
            assert torch.equal(now[others.cuda()].nan_to_num(9.0), before.flatten(0, 1)[others.cuda()].nan_to_num(9.0))
        C.check(got["attended"], *F.shared(got["turned"], self.k_pages, self.v_pages, self.table, *(torch.tensor(t, dtype=I32) for t in (starts, lengths)),
                                           self.prefix_table, self.prefix_requests, self.prefix_lengths, D ** -0.5), dtype)
        assert not got["attended"][live:].any()
        want, probs, bound = F.sample(got["logits"], self.uniform.cpu(), self.temperature, self.top_k, self.top_p)
        assert torch.equal(got["chosen"][0].cpu(), want) and bool(((got["chosen"][1].cpu().double() - probs).abs() <= bound).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_questions_and_then_tokens(ctx, dtype):
    """Chunks of different lengths, then single tokens, some requests pausing, each step from the tokens that the last one chose."""
    s = Session(ctx, dtype, [70, 33], [4, 3], room=40)
    g = torch.Generator().manual_seed(9)
    ctx.clear_bad_ids()
    chosen = None
    for news in ([9, 1, 4, 2, 7, 1, 3], [1] * 7, [1, 0, 1, 1, 0, 1, 1], [1] * 7):
        ids = torch.randint(0, VOCAB, (40,), generator=g).cuda()
        if chosen is not None:
            going = torch.tensor(news, dtype=torch.bool)
            ids[:sum(news)] = chosen[going.cuda()].long()
        s.uniform.copy_(torch.rand(7, generator=g))
        was = s.host()
        got = s.step(ids, dev(news))
        s.check(was, news, got)
        chosen = got["chosen"][0]
        assert bool((chosen >= 0).all())
    assert ctx.clear_bad_ids() == 0


def test_a_captured_step_goes_on_by_itself(ctx):
    """One graph of a whole step whose tokens are fed back in place, replayed over a page's end, against the definitions each time."""
    s = Session(ctx, torch.bfloat16, [40, 17], [3, 2], room=5)
    g = torch.Generator().manual_seed(4)
    ids, news = torch.randint(0, VOCAB, (5,), generator=g).cuda(), [1] * 5
    on = dev(news)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ctx.set_stream(side.cuda_stream)
    try:
        with torch.cuda.stream(side):
            for _ in range(2):                                    # every buffer that a step asks for is there before the capture
                ids.copy_(s.step(ids, on)["chosen"][0])
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                got = s.step(ids, on)
                ids.copy_(got["chosen"][0])
            for _ in range(18):
                s.uniform.copy_(torch.rand(5, generator=g))
                was = s.host()
                side.synchronize()
                graph.replay()
                side.synchronize()
                s.check(was, news, got)
                assert torch.equal(ids.int(), got["chosen"][0])
    finally:
        ctx.set_stream(0)
    assert s.lengths.tolist() == [20] * 5


def test_many_rows_of_logits(ctx):
    """More rows, of more than 8192 logits, than a grid has along its second axis, and than a set of launches takes."""
    rows, vocab = 70001, 8200
    x = torch.randn(1, vocab, generator=torch.Generator().manual_seed(3))
    u = torch.rand(17, generator=torch.Generator().manual_seed(5))
    many = u.repeat(-(-rows // 17))[:rows].cuda()
    for settings in ({}, dict(top_p=torch.full((17,), 0.9))):
        want, probs, bound = F.sample(x.expand(17, -1), u, **settings)
        got = ctx.sample(x.cuda().expand(rows, -1), many, **{k: v[:1].expand(rows).contiguous().cuda() for k, v in settings.items()})
        assert torch.equal(got[0].cpu(), want.repeat(-(-rows // 17))[:rows])
        assert bool(((got[1][-17:].cpu().double() - probs.roll(-(rows % 17))).abs() <= bound.roll(-(rows % 17))).all())


def test_tables_whose_rows_overlap_are_refused(ctx):
    """New pages are written into the table."""
    table = dev([[-1] * 6])
    call = lambda t: ctx.plan_pages(dev([0, 0]), dev([1, 1]), t, dev([3, 4]), dev([0]), 2, 8, 16)
    for t in (table.expand(2, 6), table[0].as_strided((2, 4), (2, 1))):
        with pytest.raises(she.SheError):
            call(t)
    assert call(table[0].as_strided((2, 3), (3, 1)))[3].tolist() == [48, 64] and table.tolist() == [[3, -1, -1, 4, -1, -1]]
    assert ctx.plan_pages(dev([0]), dev([1]), table[0].as_strided((1, 6), (0, 1)), dev([3]), dev([0]), 1, 8, 16)[3].tolist() == [48]
