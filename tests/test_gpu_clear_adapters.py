"""Adapters beside a shared projection on the GPU against their definition in 64 bits (include/she_clear.h)."""
import numpy as np
import pytest
import torch

import clear_forms as F
import paper_1906_00148_amd as she

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    with she.Context(she.TOY, 11, 64) as c:
        yield c


def dev(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def inputs(dtype, starts, which, A, r, K, N, seed=0, ranks=None):
    g = torch.Generator().manual_seed(seed)
    T = max(starts)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g) * std).to(dtype).cuda()
    return dict(x=normal(T, K), down=normal(A, r, K, std=K ** -0.5), up=normal(A, r, N, std=r ** -0.5), starts=dev(starts), which=dev(which),
                scale=(torch.rand(A, generator=g) * 2 - 0.5).cuda(), ranks=None if ranks is None else dev(ranks))


RAGGED = [0, 1, 1, 34, 98, 99, 163], [0, 1, 2, -1, 0, 2]         # an empty segment, one without an adapter, tiles that end early


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("K,N,r,ranks", [(64, 128, 8, None), (576, 1000, 16, [1, 16, 7]), (1024, 640, 17, [17, 0, 5]), (520, 136, 33, None),
                                         (128, 72, 64, [64, 3, 40]), (96, 520, 130, [130, 65, 64]), (2048, 512, 512, None),
                                         (577, 1001, 5, [5, 2, 1]), (33, 7, 40, None), (1, 1, 1, None)])
def test_against_the_definition(ctx, dtype, K, N, r, ranks):
    a = inputs(dtype, *RAGGED, 3, r, K, N, ranks=ranks)
    want, bound = F.adapters(**a)
    F.check(ctx.adapters(**a), want, bound, dtype)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("N", [512, 1003])
@pytest.mark.parametrize("base", ["same", "f32", "sums", "sums and steps", "in place"])
def test_bases(ctx, dtype, N, base):
    a = inputs(dtype, *RAGGED, 3, 12, 200, N)
    T = 163
    g = torch.Generator().manual_seed(5)
    if base == "f32":
        a["base"] = torch.randn(T, N, generator=g).cuda()
    elif base.startswith("sums"):
        a["base"] = torch.randint(-32768, 32768, (T, N), generator=g, dtype=torch.int32).cuda()
        a["step"] = (torch.rand(N, generator=g) / 4096).cuda() if base != "sums" else None
    else:
        a["base"] = torch.randn(T, N, generator=g).to(dtype).cuda()
    want, bound = F.adapters(**a)
    if base == "in place":
        a["out"] = a["base"]
    F.check(ctx.adapters(**a), want, bound, dtype, base)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shift", [8, 1])
def test_views(ctx, dtype, shift):
    """Rows of wider arrays, on 16 bytes and off them; what lies beside the result stays."""
    a = inputs(dtype, *RAGGED, 3, 9, 136, 264)
    want, bound = F.adapters(**a)
    for name in ("x", "down", "up"):
        wide = torch.full((*a[name].shape[:-1], a[name].shape[-1] + 16), float("nan"), dtype=dtype, device="cuda")
        wide[..., shift:shift + a[name].shape[-1]] = a[name]
        a[name] = wide[..., shift:shift + a[name].shape[-1]]
    wide = torch.full((163, 264 + 16), 7.0, dtype=dtype, device="cuda")
    out = wide[:, shift:shift + 264]
    F.check(ctx.adapters(**a, out=out), want, bound, dtype)
    assert bool((wide[:, :shift] == 7).all()) and bool((wide[:, shift + 264:] == 7).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_many_requests_of_a_token_each(ctx, dtype):
    S = 150
    rng = np.random.default_rng(3)
    a = inputs(dtype, list(range(S + 1)), rng.integers(-1, 40, S).tolist(), 40, 16, 256, 512, ranks=rng.integers(0, 17, 40).tolist())
    want, bound = F.adapters(**a)
    F.check(ctx.adapters(**a), want, bound, dtype)


def test_a_long_prompt(ctx):
    a = inputs(BF16, [0, 5, 3001], [1, 0], 2, 32, 1024, 2048)
    want, bound = F.adapters(**a)
    F.check(ctx.adapters(**a), want, bound, BF16)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_what_is_not_finite_stays_with_its_token_and_adapter(ctx, dtype):
    a = inputs(dtype, [0, 3, 40, 41], [0, 1, 2], 3, 10, 64, 128, ranks=[10, 4, 10])
    a["x"][1, 5] = float("inf")
    a["x"][39, 0] = float("nan")
    a["down"][2] = float("nan")
    a["up"][1, 4:] = float("nan")                                 # rows beyond the adapter's rank
    a["down"][1, 4:] = float("inf")
    want, _ = F.adapters(**a)
    got = ctx.adapters(**a).double().cpu()
    assert torch.equal(torch.isfinite(got), torch.isfinite(want))
    fine = torch.isfinite(want).all(1)
    assert fine.tolist() == [t not in (1, 39, 40) for t in range(41)]
    clean = dict(a, x=torch.nan_to_num(a["x"], nan=0.0, posinf=0.0), down=torch.nan_to_num(a["down"], nan=0.0, posinf=0.0),
                 up=torch.nan_to_num(a["up"], nan=0.0))
    want, bound = F.adapters(**clean)
    F.check(got[fine], want[fine], bound[fine], dtype)


def test_hidden_values_beyond_the_range_of_f16(ctx):
    """Hidden values of 2^20 and of 2^-30 whose results are ordinary."""
    for size in (2.0 ** 20, 2.0 ** -30):
        a = inputs(F16, [0, 20, 50], [0, 1], 2, 70, 1024, 128)
        half = size ** 0.5
        a["x"] = (a["x"].float() * min(half, 512.0)).half()
        a["down"] = (a["down"].float() * (size / min(half, 512.0))).half()
        a["scale"] = torch.full((2,), 1 / size, device="cuda")
        want, bound = F.adapters(**a)
        F.check(ctx.adapters(**a), want, bound, F16, size)
        a["scale"] = torch.ones(2, device="cuda")
        a["up"] = (a["up"].float() / 64).half()
        want, bound = F.adapters(**a)
        if size > 1:                                              # results beyond f16 are its infinities
            want = torch.where(want.abs() >= 65520, want.sign() * float("inf"), want)
            got = ctx.adapters(**a).double().cpu()
            near = ((want.abs() - 65520).abs() < 200) | (want.abs() > 65000)
            F.check(torch.where(near, 0.0, got), torch.where(near, 0.0, want), bound, F16)


def test_ids_out_of_range_are_left_out_and_counted(ctx):
    a = inputs(BF16, [0, 3, 6, 40], [7, 1, -5], 3, 8, 64, 128)
    ctx.clear_bad_ids()
    base = torch.randn(40, 128, device="cuda").bfloat16()
    want, bound = F.adapters(**a, base=base)
    F.check(ctx.adapters(**a, base=base), want, bound, BF16)
    assert ctx.clear_bad_ids() == 2 and ctx.clear_bad_ids() == 0
    # starts beyond the tokens: nothing outside the arrays is touched
    a["starts"] = dev([0, 3, 90000, -4])
    ctx.adapters(**a)
    ctx.adapters_grad(torch.randn(40, 128, device="cuda").bfloat16(), **a)
    a["starts"], a["which"] = dev([0, 40] * 20 + [0]), dev([0] * 40)
    ctx.adapters_grad(torch.randn(40, 128, device="cuda").bfloat16(), **a)
    torch.cuda.synchronize()


# ---- gradients
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("K,N,r,ranks", [(64, 128, 8, None), (576, 1000, 16, [1, 16, 7]), (264, 72, 33, [33, 0, 5]), (128, 520, 130, [130, 65, 64]),
                                         (577, 201, 5, [5, 2, 1]), (1, 1, 1, None)])
def test_gradients_against_the_definition(ctx, dtype, K, N, r, ranks):
    a = inputs(dtype, *RAGGED, 3, r, K, N, ranks=ranks)
    dy = torch.randn(163, N, generator=torch.Generator().manual_seed(9)).to(dtype).cuda()
    for got, (want, bound), name in zip(ctx.adapters_grad(dy, **a), F.adapters_grad(dy, **a), ("dx", "ddown", "dup")):
        F.check(got, want, bound, dtype, name)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("starts,which,A", [([0, 5000], [1], 2), ([0, 1100, 1101, 3600, 5000], [0, 2, 0, 1], 4),
                                            (list(range(0, 3001, 20)), [(7 * i) % 5 for i in range(150)], 5), ([0, 1], [0], 1)])
def test_gradients_of_adapters_that_many_workgroups_share(ctx, dtype, starts, which, A):
    a = inputs(dtype, starts, which, A, 20, 72, 136)
    dy = torch.randn(max(starts), 136, generator=torch.Generator().manual_seed(9)).to(dtype).cuda()
    base = torch.randn(max(starts), 72, generator=torch.Generator().manual_seed(10)).cuda()
    first = ctx.adapters_grad(dy, **a, base=base)
    for got, (want, bound), name in zip(first, F.adapters_grad(dy, **a, base=base), ("dx", "ddown", "dup")):
        F.check(got, want, bound, dtype, name)
    for got, again in zip(first, ctx.adapters_grad(dy, **a, base=base)):
        assert torch.equal(got, again)


def test_gradients_without_a_token(ctx):
    a = inputs(BF16, [0], [], 2, 8, 64, 72)
    dx, ddown, dup = ctx.adapters_grad(torch.empty(0, 72, dtype=BF16, device="cuda"), **a)
    assert dx.shape == (0, 64) and not ddown.any() and not dup.any()
    assert ctx.adapters(**a).shape == (0, 72)


def test_gradients_keep_what_is_not_finite_apart(ctx):
    """An infinite activation reaches the ranks that its adapter has and no other adapter's gradient."""
    a = inputs(BF16, [0, 20, 50], [0, 1], 2, 12, 64, 72, ranks=[5, 12])
    dy = torch.randn(50, 72, device="cuda").bfloat16()
    a["x"][3, 7] = float("inf")
    dx, ddown, dup = (t.double().cpu() for t in ctx.adapters_grad(dy, **a))
    assert torch.isfinite(dx).all() and torch.isfinite(ddown[1]).all() and torch.isfinite(dup[1]).all()
    assert not torch.isfinite(ddown[0, :5, 7]).any() and not ddown[0, 5:].any() and not dup[0, 5:].any()
    assert torch.isfinite(ddown[0][:, torch.arange(64) != 7]).all() and not torch.isfinite(dup[0, :5]).any()


def test_gradients_against_differences(ctx):
    """loss = sum(dy * out): its central differences along random directions, by the definition in 64 bits, are the gradients' products
    with the directions (the form is bilinear, so the differences are exact but for 64-bit rounding)."""
    a = inputs(F16, [0, 13, 60], [1, 0], 2, 6, 40, 48)
    g = torch.Generator().manual_seed(1)
    dy = torch.randn(60, 48, generator=g).half().cuda()
    grads = dict(zip(("x", "down", "up"), ctx.adapters_grad(dy, **a)))

    def loss(**changed):
        return float((F.cpu(dy) * F.adapters(**dict(a, **changed))[0]).sum())
    for name, grad in grads.items():
        t = F.cpu(a[name])
        for _ in range(3):
            d = torch.randn(t.shape, generator=g, dtype=torch.float64)
            # F.adapters takes the roundoff from the type; the values may be wider
            moved = [t + s * 0.25 * d for s in (1, -1)]
            F.UNIT[torch.float64], F.SPLIT[torch.float64] = 0.0, 0.0
            slope = (loss(**{name: moved[0]}) - loss(**{name: moved[1]})) / 0.5
            # rounding of the gradient's elements, independent of each other: six of its standard deviations
            allowed = 6 * F.UNIT[F16] * float((F.cpu(grad) * d).norm()) + 1e-9 * abs(slope)
            assert abs(slope - float((F.cpu(grad) * d).sum())) <= allowed, name


# ---- streams
def test_on_another_stream_and_in_a_graph(ctx):
    a = inputs(BF16, *RAGGED, 3, 12, 512, 512)
    dy = torch.randn(163, 512, device="cuda").bfloat16()
    want = [ctx.adapters(**a), *ctx.adapters_grad(dy, **a)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a["x"] = a["x"] + 0                                       # made on that stream just before
        got = [ctx.adapters(**a), *ctx.adapters_grad(dy, **a)]
        total = sum(t.float().sum() for t in got)                 # and read on it just after
    side.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want)) and torch.isfinite(total)
    with torch.cuda.graph(torch.cuda.CUDAGraph()):                # the context's stream is the default one: it cannot be captured
        with pytest.raises(she.SheError):
            ctx.adapters(**a)
    ctx.set_stream(side.cuda_stream)
    try:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = [ctx.adapters(**a), *ctx.adapters_grad(dy, **a)]
        for k in range(3):
            a["x"].copy_(torch.randn_like(a["x"]))
            want = [ctx.adapters(**a), *ctx.adapters_grad(dy, **a)]
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(g, w) for g, w in zip(got, want)), k
    finally:
        ctx.set_stream(0)


def test_refusals(ctx):
    a = inputs(BF16, [0, 4], [0], 1, 8, 64, 72)

    def refused(code, **changed):
        with pytest.raises(she.SheError) as e:
            ctx.adapters(**dict(a, **changed))
        assert e.value.code == code, e.value
    refused(-1, x=a["x"].float())
    refused(-1, x=a["x"].cpu())
    refused(-1, x=a["x"].T)
    refused(-1, down=a["down"].half())
    refused(-1, down=a["down"][:, :4])
    refused(-1, starts=a["starts"].long())
    refused(-1, starts=a["starts"][:1])
    refused(-1, scale=a["scale"].double())
    refused(-1, ranks=dev([1, 2]))
    refused(-1, base=torch.zeros(4, 71, device="cuda"))
    refused(-1, base=torch.zeros(4, 72, device="cuda", dtype=torch.float64))
    refused(-1, base=torch.zeros(4, 72, device="cuda"), step=torch.ones(72, device="cuda"))
    refused(-1, out=torch.zeros(4, 72, device="cuda"))
    big = torch.zeros(1, 513, 8, dtype=BF16, device="cuda")
    refused(-4, x=a["x"][:, :8], down=big, up=big)
    with pytest.raises(she.SheError):
        ctx.adapters_grad(torch.zeros(4, 72, device="cuda", dtype=BF16), **a, base=torch.zeros(4, 64, device="cuda", dtype=torch.int32))
