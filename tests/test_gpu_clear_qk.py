"""Norms and rotation of queries and keys on the GPU against their definition in 64 bits (include/she_clear.h)."""
import pytest
import torch

import clear_forms as F
import paper_1906_00148_amd as she

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16
EPS = 1e-6


@pytest.fixture(scope="module")
def ctx():
    with she.Context(she.TOY, 12, 64) as c:
        yield c


def inputs(dtype, T, Hq, Hkv, D, rot, places=50, seed=0, weights=True):
    g = torch.Generator().manual_seed(seed)
    angle = torch.rand(places, rot // 2, generator=g) * 6.3
    w = [(torch.randn(D, generator=g) * 0.3 + 1).cuda() if weights else None for _ in range(2)]
    return dict(q=torch.randn(T, Hq, D, generator=g).to(dtype).cuda(), k=torch.randn(T, Hkv, D, generator=g).to(dtype).cuda(), wq=w[0], wk=w[1],
                cos=angle.cos().cuda(), sin=angle.sin().cuda(), positions=torch.randint(0, places, (T,), generator=g, dtype=torch.int32).cuda())


SHAPES = [(1, 1, 1, 8, 8), (5, 8, 2, 64, 64), (33, 32, 8, 128, 128), (7, 3, 3, 80, 40), (9, 7, 1, 96, 32), (4, 4, 2, 256, 256), (3, 2, 1, 512, 64),
          (6, 5, 2, 36, 20), (5, 3, 1, 37, 36), (2, 2, 2, 128, 0), (11, 2, 1, 64, 18), (700, 12, 4, 64, 64)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,D,rot", SHAPES)
def test_against_the_definition(ctx, dtype, interleaved, T, Hq, Hkv, D, rot):
    a = inputs(dtype, T, Hq, Hkv, D, rot, weights=T != 5)
    qo, ko = ctx.qk_rotate(**a, eps=EPS, interleaved=interleaved)
    for got, x, w in ((qo, a["q"], a["wq"]), (ko, a["k"], a["wk"])):
        want, bound = F.rotate(x, w, a["cos"], a["sin"], a["positions"], EPS, interleaved)
        F.check(got, want, bound, dtype)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,D,rot", SHAPES + [(9000, 4, 2, 16, 16)])
def test_gradients_against_the_definition(ctx, dtype, interleaved, T, Hq, Hkv, D, rot):
    a = inputs(dtype, T, Hq, Hkv, D, rot, weights=T != 5)
    g = torch.Generator().manual_seed(4)
    dq, dk = (torch.randn(t.shape, generator=g).to(dtype).cuda() for t in (a["q"], a["k"]))
    got = ctx.qk_rotate_grad(dq, dk, **a, eps=EPS, interleaved=interleaved)
    for x, dy, w, dx, dw in ((a["q"], dq, a["wq"], got[0], got[2]), (a["k"], dk, a["wk"], got[1], got[3])):
        (want, bound), (want_w, bound_w) = F.rotate_grad(dy, x, w, a["cos"], a["sin"], a["positions"], EPS, interleaved)
        F.check(dx, want, bound, dtype)
        F.check(dw, want_w, bound_w, torch.float32)
    again = ctx.qk_rotate_grad(dq, dk, **a, eps=EPS, interleaved=interleaved)
    assert all(torch.equal(x, y) for x, y in zip(got, again))


def test_gradients_against_differences(ctx):
    """loss = sum(dq' * q'): central differences of the definition in 64 bits."""
    a = inputs(F16, 6, 3, 1, 24, 16)
    g = torch.Generator().manual_seed(2)
    dq, dk = (torch.randn(t.shape, generator=g).half().cuda() for t in (a["q"], a["k"]))
    grads = ctx.qk_rotate_grad(dq, dk, **a, eps=EPS)

    def loss(q, wq):
        return float((F.cpu(dq) * F.rotate(q, wq, a["cos"], a["sin"], a["positions"], EPS, False)[0]).sum())
    q, w, h = F.cpu(a["q"]), F.cpu(a["wq"]), 1e-5
    for _ in range(4):
        d, e = torch.randn(q.shape, generator=g, dtype=torch.float64), torch.randn(w.shape, generator=g, dtype=torch.float64)
        slope = (loss(q + h * d, w) - loss(q - h * d, w)) / (2 * h)
        # six standard deviations of the roundings, and the differences' own h^2 and 2^-52 / h
        assert abs(slope - float((F.cpu(grads[0]) * d).sum())) <= 6 * F.UNIT[F16] * float((F.cpu(grads[0]) * d).norm()) + 1e-6 * (1 + abs(slope))
        slope = (loss(q, w + h * e) - loss(q, w - h * e)) / (2 * h)
        assert abs(slope - float((F.cpu(grads[2]) * e).sum())) <= 2e-5 * float((F.cpu(grads[2]) * e).abs().sum()) + 1e-6 * (1 + abs(slope))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shift", [8, 1])
def test_views_of_one_projection_and_in_place(ctx, dtype, shift):
    T, Hq, Hkv, D = 21, 6, 2, 72
    a = inputs(dtype, T, Hq, Hkv, D, 72)
    row = torch.full((T, shift + (Hq + Hkv) * D + 8), 5.0, dtype=dtype, device="cuda")
    q, k = row[:, shift:shift + Hq * D].unflatten(1, (Hq, D)), row[:, shift + Hq * D:shift + (Hq + Hkv) * D].unflatten(1, (Hkv, D))
    q.copy_(a["q"]), k.copy_(a["k"])
    want = ctx.qk_rotate(**a)
    dq, dk = torch.randn_like(a["q"]), torch.randn_like(a["k"])
    want_grad = ctx.qk_rotate_grad(dq, dk, **a)
    got_grad = ctx.qk_rotate_grad(dq, dk, **dict(a, q=q, k=k))
    assert all(torch.equal(x, y) for x, y in zip(got_grad, want_grad))
    got = ctx.qk_rotate(**dict(a, q=q, k=k), out=(q, k))
    assert torch.equal(got[0], want[0]) and torch.equal(k, want[1])
    assert bool((row[:, :shift] == 5).all()) and bool((row[:, -8:] == 5).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("page", [1, 16, 7])
@pytest.mark.parametrize("T,Hq,Hkv,D,rot", [(1, 1, 1, 8, 8), (33, 32, 8, 128, 128), (13, 4, 4, 80, 40), (5, 6, 2, 36, 20)])
def test_into_pages(ctx, dtype, page, T, Hq, Hkv, D, rot):
    a = inputs(dtype, T, Hq, Hkv, D, rot)
    g = torch.Generator().manual_seed(6)
    pages = T // page + 3
    v = torch.randn(T, Hkv, D, generator=g).to(dtype).cuda()
    both = torch.randn(pages, 2, page, Hkv, D, generator=g).to(dtype).cuda()       # keys and values of a page side by side
    before = both.clone()
    slots = torch.randperm(pages * page, generator=g)[:T]
    slots[T // 2] = -1
    qo, ko = ctx.qk_rotate(**a)
    got = ctx.qk_rotate_append(a["q"], a["k"], v, a["wq"], a["wk"], a["cos"], a["sin"], a["positions"], both[:, 0], both[:, 1], slots.cuda())
    assert torch.equal(got, qo)
    for t in range(T):
        if slots[t] >= 0:
            p, i = int(slots[t]) // page, int(slots[t]) % page
            before[p, 0, i], before[p, 1, i] = ko[t], v[t]
    assert torch.equal(both, before)


def test_ids_out_of_range_are_left_out_and_counted(ctx):
    a = inputs(BF16, 40, 4, 2, 64, 64)
    a["positions"][3], a["positions"][9] = 50, -1
    ctx.clear_bad_ids()
    qo, ko = ctx.qk_rotate(**a)
    want, bound = F.rotate(a["q"], a["wq"], a["cos"], a["sin"], a["positions"], EPS, False)
    F.check(qo, want, bound, BF16)
    assert not qo[3].any() and not ko[9].any() and ctx.clear_bad_ids() == 2
    grads = ctx.qk_rotate_grad(qo, ko, **a)
    assert not grads[0][3].any() and not grads[1][9].any() and ctx.clear_bad_ids() == 2
    k_pages, v_pages = torch.zeros(2, 2, 32, 2, 64, dtype=BF16, device="cuda")
    slots = torch.arange(40, device="cuda")
    slots[0], slots[1] = 64, -7
    got = ctx.qk_rotate_append(a["q"], a["k"], a["k"], a["wq"], a["wk"], a["cos"], a["sin"], a["positions"], k_pages, v_pages, slots)
    assert torch.equal(got, qo) and ctx.clear_bad_ids() == 4
    for t in (0, 1, 3, 9):
        assert not k_pages.flatten(0, 1)[t].any() and not v_pages.flatten(0, 1)[t].any()
    assert torch.equal(k_pages.flatten(0, 1)[10:40], ko[10:])


def test_what_is_not_finite_stays_in_its_head(ctx):
    a = inputs(BF16, 6, 4, 2, 64, 32)
    clean = ctx.qk_rotate(**a)
    a["q"][2, 1, 40] = float("inf")
    a["k"][4, 0, 1] = float("nan")
    qo, ko = ctx.qk_rotate(**a)
    assert bool(torch.isnan(ko[4, 0]).all()) and torch.equal(ko[:4], clean[1][:4]) and torch.equal(ko[4, 1], clean[1][4, 1])
    assert bool(torch.isnan(qo[2, 1, 40])) and torch.equal(qo[2, 0], clean[0][2, 0]) and torch.equal(qo[2, 2:], clean[0][2, 2:])
    a = inputs(BF16, 3, 2, 1, 64, 64)
    a["q"][1] = 0
    qo, _ = ctx.qk_rotate(**a)
    assert not qo[1].any()


def test_nothing_to_do(ctx):
    a = inputs(BF16, 0, 2, 1, 64, 64)
    qo, ko = ctx.qk_rotate(**a)
    assert qo.shape == (0, 2, 64) and ko.shape == (0, 1, 64)
    dq, dk, dwq, dwk = ctx.qk_rotate_grad(qo, ko, **a)
    assert dq.shape == (0, 2, 64) and not dwq.any() and not dwk.any()


def test_on_another_stream_and_in_a_graph(ctx):
    a = inputs(BF16, 70, 8, 2, 128, 128)
    want = [*ctx.qk_rotate(**a), *ctx.qk_rotate_grad(a["q"], a["k"], **a)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a["q"] = a["q"] + 0
        got = [*ctx.qk_rotate(**a), *ctx.qk_rotate_grad(a["q"], a["k"], **a)]
        total = sum(t.float().sum() for t in got)
    side.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want)) and torch.isfinite(total)
    with torch.cuda.graph(torch.cuda.CUDAGraph()):                # the context's stream is the default one: it cannot be captured
        with pytest.raises(she.SheError):
            ctx.qk_rotate(**a)
    ctx.set_stream(side.cuda_stream)
    try:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = [*ctx.qk_rotate(**a), *ctx.qk_rotate_grad(a["q"], a["k"], **a)]
        for k in range(3):
            a["q"].copy_(torch.randn_like(a["q"]))
            want = [*ctx.qk_rotate(**a), *ctx.qk_rotate_grad(a["q"], a["k"], **a)]
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(g, w) for g, w in zip(got, want)), k
    finally:
        ctx.set_stream(0)


def test_refusals(ctx):
    a = inputs(BF16, 4, 2, 1, 64, 32)

    def refused(code, **changed):
        with pytest.raises(she.SheError) as e:
            ctx.qk_rotate(**dict(a, **changed))
        assert e.value.code == code, e.value
    refused(-1, q=a["q"].float())
    refused(-1, k=a["k"].half())
    refused(-1, k=a["k"][:, :, :32])
    refused(-1, q=a["q"].transpose(1, 2).contiguous().transpose(1, 2))
    refused(-1, wq=a["wq"].bfloat16())
    refused(-1, cos=a["cos"][:, :8])
    refused(-1, cos=a["cos"].cpu())
    refused(-1, positions=a["positions"].long())
    refused(-1, eps=-1.0)
    refused(-1, cos=torch.zeros(4, 40, device="cuda"), sin=torch.zeros(4, 40, device="cuda"))
    wide = torch.zeros(4, 2, 520, dtype=BF16, device="cuda")
    refused(-4, q=wide, k=wide, wq=None, wk=None)
    pages = torch.zeros(2, 2, 16, 1, 64, dtype=BF16, device="cuda")
    rest = (a["wq"], a["wk"], a["cos"], a["sin"], a["positions"])
    slots = torch.zeros(4, dtype=torch.int64, device="cuda")
    for args in ((pages[0], pages[1, :, :8], slots), (pages[0], pages[1].half(), slots), (pages[0], pages[1], slots.int()),
                 (pages[0], pages[1].transpose(0, 1).contiguous().transpose(0, 1), slots)):
        with pytest.raises(she.SheError):
            ctx.qk_rotate_append(a["q"], a["k"], a["k"], *rest, *args)
