"""The choice of the next token on the GPU against its definition in 64 bits (include/she_clear.h)."""
import pytest
import torch

import clear_step_forms as F
import paper_1906_00148_amd as she

pytestmark = pytest.mark.gpu
BF16, F16, F32, SUMS = torch.bfloat16, torch.float16, torch.float32, torch.int32
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ctx():
    with she.Context(she.TOY, 21, 64) as c:
        yield c


def compare(ctx, logits, uniform, **settings):
    """The kernel's answers are the definition's."""
    want, probs, bound = F.sample(logits, uniform, **settings)
    on = {k: v.cuda() for k, v in settings.items()}
    tokens, got = ctx.sample(logits.cuda(), uniform.cuda(), **on)
    assert tokens.dtype is torch.int32 and got.dtype is torch.float32
    assert torch.equal(tokens.cpu(), want), (tokens.cpu(), want)
    assert bool(((got.cpu().double() - probs).abs() <= bound).all()), (got.cpu(), probs)
    return tokens, got


def numbers(rows, vocab, dtype, seed=0, spread=2.5):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, vocab, generator=g) * spread
    x[:, ::max(1, vocab // 13)] += 6
    if dtype is SUMS:
        return (x * 300).round().to(SUMS), dict(step=(torch.rand(vocab, generator=g) + 0.5) / 300), g
    return x.to(dtype), {}, g


def each(rows, values, dtype=torch.float32):
    return torch.tensor([values[r % len(values)] for r in range(rows)], dtype=dtype)


VOCABS = [1, 2, 7, 8, 9, 511, 512, 513, 4095, 8191, 8200, 32001, 65537, 131072]


@pytest.mark.parametrize("dtype", [BF16, F16, F32, SUMS])
@pytest.mark.parametrize("vocab", VOCABS)
def test_without_filters(ctx, dtype, vocab):
    x, step, g = numbers(9, vocab, dtype, vocab)
    compare(ctx, x, torch.rand(9, generator=g), **step)
    compare(ctx, x, torch.rand(9, generator=g), temperature=each(9, [0.3, 1.0, 1.7, 0.0, 25.0]), **step)


@pytest.mark.parametrize("dtype", [BF16, F16, F32, SUMS])
@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("filters", ["k", "p", "min", "all"])
def test_filters(ctx, dtype, vocab, filters):
    rows = 24
    x, step, g = numbers(rows, vocab, dtype, vocab + 1)
    a = dict(step, temperature=each(rows, [0.7, 1.0, 1.3, 6.0]))
    if filters in ("k", "all"):
        a["top_k"] = each(rows, [1, 2, 50, 1000, 0, vocab - 1, vocab, vocab + 1, 5, -3, 20000], torch.int32)
    if filters in ("p", "all"):
        a["top_p"] = each(rows, [0.9, 0.5, 0.01, 0.999, 1.0, 0.0, 0.95])
    if filters in ("min", "all"):
        a["min_p"] = each(rows, [0.1, 0.0, 0.5, 1e-6, 1.0])
    compare(ctx, x, torch.rand(rows, generator=g), **a)


@pytest.mark.parametrize("dtype", [BF16, F32, SUMS])
@pytest.mark.parametrize("vocab", [5000, 40000])
@pytest.mark.parametrize("shift", [-60.0, 0.0, 60.0])
def test_a_top_p_of_thousands_and_a_min_p_of_few(ctx, dtype, vocab, shift):
    """Flat rows: the border of either filter lies far behind, before or beside the other's."""
    rows = 20
    g = torch.Generator().manual_seed(vocab)
    x, step = torch.randn(rows, vocab, generator=g) * 1.5 + shift, {}
    if dtype is SUMS:
        x, step = (x * 500).round().to(SUMS), dict(step=torch.full((vocab,), 1 / 500))
    else:
        x = x.to(dtype)
    p, m = each(rows, [0.9, 0.999, 0.5, 0.99]), each(rows, [0.5, 1e-3, 0.05, 0.9, 1e-5])
    u = torch.rand(rows, generator=g)
    u[::4] = 1.0
    compare(ctx, x, u, top_p=p, min_p=m, **step)
    compare(ctx, x, u, top_p=p, min_p=m, top_k=each(rows, [0, 5000, 300], torch.int32), **step)


@pytest.mark.parametrize("rows", [1, 2, 3, 5, 17, 64, 255, 300])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_numbers_of_rows(ctx, rows, dtype):
    x, step, g = numbers(rows, 20011, dtype, rows)
    u = torch.rand(rows, generator=g)
    compare(ctx, x, u)
    compare(ctx, x, u, temperature=each(rows, [0.8, 1.2]), top_k=each(rows, [40, 0, 3000], torch.int32), top_p=each(rows, [0.9, 1.0]))


def test_the_largest_vocabulary(ctx):
    x, _, g = numbers(3, 1 << 20, BF16)
    a = dict(temperature=torch.tensor([1.0, 1.0, 3.0]), top_k=torch.tensor([0, 7000, 0], dtype=torch.int32), top_p=torch.tensor([1.0, 0.9, 0.7]))
    compare(ctx, x, torch.rand(3, generator=g), **a)
    compare(ctx, x, torch.rand(3, generator=g))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("vocab", [10, 600, 40000])
def test_equal_logits(ctx, dtype, vocab):
    """Ties everywhere: the lower index comes first, and a border that falls on a token exactly does not move."""
    rows = 12
    u = each(rows, [0.0, 0.25, 0.5, 0.75, 0.999999])
    for x in (torch.zeros(rows, vocab), torch.full((rows, vocab), -7.5), torch.arange(vocab).remainder(3).float().repeat(rows, 1),
              torch.arange(vocab).remainder(2).float().mul(-0.0).repeat(rows, 1)):
        x = x.to(dtype)
        compare(ctx, x, u)
        compare(ctx, x, u, top_k=each(rows, [1, 3, vocab // 2, vocab - 1], torch.int32))
        compare(ctx, x, u, top_p=each(rows, [0.5, 0.25, 0.125, 0.75]))
        compare(ctx, x, u, top_k=each(rows, [8, vocab // 2], torch.int32), top_p=each(rows, [0.5, 0.25, 0.75]), min_p=each(rows, [0.0, 1.0]))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_masked_and_special_logits(ctx, dtype):
    """Rows of which a mask leaves few tokens, one or none; the type's lowest and largest values; infinities and NaN."""
    vocab = 3000
    x, _, g = numbers(12, vocab, dtype)
    info = torch.finfo(dtype)
    x[0] = -INF
    x[1] = NAN
    x[2], x[2, 1234] = -INF, -80.0
    x[3, torch.randperm(vocab, generator=g)[:2900]] = -INF
    x[4, 5::7] = NAN
    x[5, [17, 400, 2999]] = INF
    x[6] = info.min
    x[7], x[7, 77] = info.min, info.max
    x[8] = info.max
    x[9, ::2] = info.min
    x[10, :] = NAN
    x[10, 2998] = INF
    x[11] = torch.where(torch.arange(vocab) % 2 == 0, info.tiny, -info.tiny)
    for u in (0.0, 0.37, 0.99):
        u = torch.full((12,), u)
        compare(ctx, x, u)
        for T in (0.0, -1.0, NAN, 1e-38, 1e-45, 0.01, 1e9, INF):
            compare(ctx, x, u, temperature=torch.full((12,), T))
        for T in (0.5, INF, 1e-38):
            compare(ctx, x, u, temperature=torch.full((12,), T), top_k=torch.full((12,), 60, dtype=torch.int32), top_p=torch.full((12,), 0.6))
            compare(ctx, x, u, temperature=torch.full((12,), T), top_p=torch.full((12,), 0.6), min_p=torch.full((12,), 0.3))
            compare(ctx, x, u, temperature=torch.full((12,), T), min_p=torch.full((12,), 2.0))


def test_settings_at_their_ends(ctx):
    x, _, g = numbers(8, 5000, F32)
    u = torch.tensor([0.0, 1.0, 2.0, -1.0, NAN, INF, 1 - 2.0 ** -24, 2.0 ** -149])
    compare(ctx, x, u)
    compare(ctx, x, u, top_p=torch.tensor([NAN, INF, -INF, -1.0, 1.0, 0.0, 1 - 2.0 ** -24, 2.0 ** -149]))
    compare(ctx, x, u, min_p=torch.tensor([NAN, INF, -INF, -1.0, 1.0, 0.0, 1 - 2.0 ** -24, 2.0 ** -149]))
    compare(ctx, x, u, top_k=torch.tensor([0, -1, -2 ** 31, 2 ** 31 - 1, 5000, 4999, 1, 2], dtype=torch.int32))


@pytest.mark.parametrize("dtype", [F32, SUMS])
def test_logits_that_differ_in_their_last_bits(ctx, dtype):
    """A bin of the histogram that holds all of the row, and one that has zero in its middle."""
    rows, vocab = 8, 30000
    g = torch.Generator().manual_seed(5)
    x = 9 + torch.randn(rows, vocab, generator=g) * 1e-5
    x[4:] = torch.randn(4, vocab, generator=g) * 10.0 ** torch.randint(-38, -2, (4, vocab), generator=g).float()
    step = {}
    if dtype is SUMS:
        x, step = (x[:4] * 1e7).round().to(SUMS).repeat(2, 1), dict(step=torch.full((vocab,), 1e-7))
    k, p = each(rows, [100, 29000, 0, 15000], torch.int32), each(rows, [0.5, 1.0, 0.3])
    compare(ctx, x, torch.rand(rows, generator=g), top_k=k, top_p=p, **step)


@pytest.mark.parametrize("dtype", [BF16, F32, SUMS])
@pytest.mark.parametrize("at", [0, 1, 5])
def test_rows_of_a_wider_array(ctx, dtype, at):
    x, step, g = numbers(6, 1001, dtype)
    wide = torch.full((6, 1200), 100, dtype=dtype, device="cuda")
    wide[:, at:at + 1001] = x.cuda()
    u = torch.rand(6, generator=g)
    a = dict(step, top_k=each(6, [0, 30], torch.int32), top_p=each(6, [0.9, 0.8, 1.0]))
    on = {k: v.cuda() for k, v in a.items()}
    want = ctx.sample(x.cuda(), u.cuda(), **on)
    out = torch.empty(6, dtype=torch.int32, device="cuda"), torch.empty(6, device="cuda")
    got = ctx.sample(wide[:, at:at + 1001], u.cuda(), out=out, **on)
    assert got[0] is out[0] and all(torch.equal(g, w) for g, w in zip(got, want))
    # every row the same memory
    got = ctx.sample(x[:1].cuda().expand(6, -1), u.cuda(), **on)
    assert torch.equal(got[0].cpu(), F.sample(x[:1].expand(6, -1), u, **a)[0])


def test_draws_follow_the_weights(ctx):
    """Evenly spread numbers give every token its share, to one draw."""
    x = torch.tensor([[1.0, -INF, 0.0, 2.0, 0.5, -1.0]])
    n = 4096
    u = (torch.arange(n) + 0.5) / n
    tokens, probs = ctx.sample(x.cuda().expand(n, -1), u.cuda())
    share = torch.softmax(x[0].double(), 0)
    count = torch.bincount(tokens.cpu(), minlength=6)
    assert bool(((count - share * n).abs() <= 1).all()) and count[1] == 0
    assert torch.equal(probs.cpu(), share[tokens.cpu().long()].float())


def test_on_another_stream_and_in_a_graph(ctx):
    x, _, g = numbers(5, 30011, BF16)
    x, u = x.cuda(), torch.rand(5, generator=g).cuda()
    a = dict(temperature=each(5, [0.8, 1.5]).cuda(), top_k=each(5, [0, 200], torch.int32).cuda(), top_p=each(5, [0.9, 1.0]).cuda())
    want = ctx.sample(x, u, **a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ctx.sample(x, u, **a)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(g, w) for g, w in zip(got, want))
    ctx.set_stream(side.cuda_stream)
    try:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            ctx.sample(x, u, **a)
            side.synchronize()
            with torch.cuda.graph(graph, stream=side):
                out = ctx.sample(x, u, **a)
    finally:
        ctx.set_stream(0)
    for seed in (None, 3, 4):
        if seed:
            u.copy_(torch.rand(5, generator=torch.Generator().manual_seed(seed)))
            want = ctx.sample(x, u, **a)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(out, want))


def test_refusals(ctx):
    x, u = torch.zeros(2, 8, device="cuda"), torch.zeros(2, device="cuda")
    for bad in (dict(logits=x.double()), dict(logits=x.mT.contiguous().mT), dict(logits=x.cpu()), dict(uniform=u[:1]), dict(uniform=u.double()), dict(uniform=None),
                dict(step=torch.ones(8, device="cuda")), dict(logits=x.int(), step=torch.ones(7, device="cuda")), dict(top_k=u), dict(top_p=u.half()),
                dict(temperature=torch.ones(3, device="cuda")), dict(min_p=torch.ones(2)), dict(logits=x[:, :0]),
                dict(logits=torch.zeros(1, (1 << 20) + 1, dtype=BF16, device="cuda"), uniform=u[:1])):
        with pytest.raises(she.SheError):
            ctx.sample(**{**dict(logits=x, uniform=u), **bad})
    assert ctx.sample(x[:0], u[:0])[0].shape == (0,)


def test_gradients_are_not_lost_in_silence(ctx):
    x, u = torch.zeros(2, 8, device="cuda", requires_grad=True), torch.zeros(2, device="cuda")
    tokens, probs = ctx.sample(x, u)
    assert not tokens.requires_grad
    with pytest.raises(she.SheError):
        probs.sum().backward()
