"""What torch's automatic differentiation sees of the clear side's calls: no gradient is lost in silence, no write goes unseen."""
import pytest
import torch

import paper_1906_00148_amd as she

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
I32 = torch.int32


@pytest.fixture(scope="module")
def ctx():
    with she.Context(she.TOY, 17, 64) as c:
        yield c


def adapters():
    torch.manual_seed(1)
    half = lambda *size: torch.randn(*size, device="cuda").to(BF16)
    return dict(x=half(3, 16), down=half(2, 4, 16), up=half(2, 4, 24), starts=torch.tensor([0, 1, 3], dtype=I32, device="cuda"),
                which=torch.tensor([1, 0], dtype=I32, device="cuda"), scale=torch.ones(2, device="cuda"))


def heads():
    torch.manual_seed(2)
    half = lambda *size: torch.randn(*size, device="cuda").to(BF16)
    return dict(q=half(3, 2, 8), k=half(3, 1, 8), wq=torch.ones(8, device="cuda"), wk=torch.ones(8, device="cuda"), cos=torch.ones(5, 4, device="cuda"),
                sin=torch.zeros(5, 4, device="cuda"), positions=torch.tensor([0, 1, 2], dtype=I32, device="cuda"))


def cache():
    half = lambda *size: torch.randn(*size, device="cuda").to(BF16)
    return dict(k_pages=half(4, 16, 1, 8), v_pages=half(4, 16, 1, 8))


def results(ctx, call, a):
    r = getattr(ctx, call)(**a)
    return r if isinstance(r, tuple) else (r,)


def every_call():
    tokens = dict(table=torch.zeros(1, 4, dtype=I32, device="cuda"), starts=torch.tensor([0, 3], dtype=I32, device="cuda"),
                  lengths=torch.tensor([20], dtype=I32, device="cuda"))
    half = lambda *size: torch.randn(*size, device="cuda").to(BF16)
    return [("adapters", adapters(), ("x", "down", "up", "scale", "base")), ("qk_rotate", heads(), ("q", "k", "wq", "wk")),
            ("qk_rotate_append", dict(heads(), v=half(3, 1, 8), **cache(), slots=torch.tensor([5, 6, 7], device="cuda")), ("q", "k", "v", "wk")),
            ("attend_pages", dict(cache(), q=half(3, 2, 8), **tokens), ("q", "k_pages", "v_pages")),
            ("adapters_grad", dict(adapters(), dy=half(3, 24)), ("dy", "x", "down")), ("qk_rotate_grad", dict(heads(), dq_out=half(3, 2, 8), dk_out=half(3, 1, 8)), ("dq_out", "q"))]


@pytest.mark.parametrize("index", range(6))
def test_a_gradient_that_is_not_recorded_raises(ctx, index):
    call, a, names = every_call()[index]
    if call == "adapters":
        a["base"] = torch.zeros(3, 24, device="cuda")
    want = results(ctx, call, a)
    assert not any(t.requires_grad for t in want)
    for name in names:
        b = dict(a, **{name: a[name].clone().requires_grad_()})
        got = results(ctx, call, b)
        assert all(torch.equal(g, w) for g, w in zip(got, want))
        for t in got:
            assert t.requires_grad
            with pytest.raises(she.SheError):
                t.float().sum().backward(retain_graph=True)
        assert b[name].grad is None
        with torch.no_grad():
            got = results(ctx, call, b)
        assert all(torch.equal(g, w) and not g.requires_grad for g, w in zip(got, want))


def test_a_function_that_joins_the_calls_has_gradients(ctx):
    a = adapters()

    class Joined(torch.autograd.Function):
        @staticmethod
        def forward(f, x, down, up):
            f.save_for_backward(x, down, up)
            return ctx.adapters(x, down, up, a["starts"], a["which"], a["scale"])

        @staticmethod
        def backward(f, dy):
            return ctx.adapters_grad(dy.contiguous(), *f.saved_tensors, a["starts"], a["which"], a["scale"])
    leaves = [a[n].clone().requires_grad_() for n in ("x", "down", "up")]
    dy = torch.randn(3, 24, device="cuda").to(BF16)
    got = torch.autograd.grad(Joined.apply(*leaves), leaves, dy)
    want = ctx.adapters_grad(dy, **a)
    assert all(torch.equal(g, w) for g, w in zip(got, want))


def test_what_a_call_writes_counts_as_changed(ctx):
    """A tensor that backward needs as it was, written over in between: torch notices."""
    w = torch.ones((), device="cuda", requires_grad=True)

    def written_over(t, write):
        loss = (t.float() if t.dtype is torch.float32 else t).mul(w.to(t.dtype)).sum()
        write()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    a = adapters()
    out = torch.zeros(3, 24, dtype=BF16, device="cuda")
    written_over(out, lambda: ctx.adapters(**a, out=out))
    h = heads()
    q, k = torch.zeros_like(h["q"]), torch.zeros_like(h["k"])
    written_over(q, lambda: ctx.qk_rotate(**h, out=(q, k)))
    written_over(k, lambda: ctx.qk_rotate(**h, out=(q, k)))
    c = cache()
    append = dict(h, v=h["k"], **c, slots=torch.tensor([5, 6, 7], device="cuda"))
    written_over(c["k_pages"], lambda: ctx.qk_rotate_append(**append))
    written_over(c["v_pages"], lambda: ctx.qk_rotate_append(**append))
    written_over(q, lambda: ctx.qk_rotate_append(**append, out=q))
    tokens = dict(table=torch.zeros(1, 4, dtype=I32, device="cuda"), starts=torch.tensor([0, 3], dtype=I32, device="cuda"),
                  lengths=torch.tensor([20], dtype=I32, device="cuda"))
    written_over(q, lambda: ctx.attend_pages(h["q"], **c, **tokens, out=q))
    with torch.inference_mode():
        out = torch.zeros(3, 24, dtype=BF16, device="cuda")
        assert torch.equal(ctx.adapters(**a, out=out), ctx.adapters(**a))
