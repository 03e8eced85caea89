"""Forward-mode differentiation through the clear side's calls, without a GPU: a tangent is refused and not lost in silence."""
import pytest
import torch
import torch.autograd.forward_ad as forward

import paper_1906_00148_amd as she
from paper_1906_00148_amd import clear
from test_host_clear_binding import arguments as older_arguments, library  # noqa: F401

# what a result follows smoothly or a call writes into
TENSORS = {"adapters": "x down up scale base step out", "adapters_grad": "dy x down up scale base", "qk_rotate": "q k wq wk cos sin",
           "qk_rotate_append": "q k v wq wk cos sin k_pages v_pages out", "qk_rotate_grad": "dq_out dk_out q k wq wk cos sin",
           "attend_pages": "q k_pages v_pages out", "attend_shared": "q k_pages v_pages out", "sample": "logits temperature"}


def arguments():
    a = older_arguments()
    i32 = torch.int32
    a["adapters"].update(base=torch.zeros(3, 24))
    del a["adapters"]["step"]
    a["attend_shared"] = dict(a["attend_pages"], prefix_table=torch.zeros(1, 4, dtype=i32), prefix_requests=torch.zeros(2, dtype=i32),
                              prefix_lengths=torch.zeros(1, dtype=i32))
    a["sample"] = dict(logits=torch.zeros(2, 9), uniform=torch.zeros(2), temperature=torch.ones(2), top_k=torch.zeros(2, dtype=i32), top_p=torch.ones(2))
    return a


@pytest.fixture
def ctx(library, monkeypatch):  # noqa: F811
    library.device = -1                                            # what tensors in host memory say
    monkeypatch.setattr(clear.Calls, "_call", lambda self, fn, args: fn(self._h, args))
    with she.Context(she.TOY, 1, 16, use_torch_pool=False) as c:
        yield c


def names(call, a):
    return [n for n in TENSORS[call].split() if n in a]


@pytest.mark.parametrize("call", sorted(TENSORS))
def test_a_tangent_is_refused(library, ctx, call):  # noqa: F811
    a = arguments()[call]
    for name in names(call, a):
        with forward.dual_level():
            b = dict(a, **{name: forward.make_dual(a[name], torch.ones_like(a[name]))})
            with pytest.raises(she.SheError, match="tangent"):
                getattr(ctx, call)(**b)
            assert not [n for n, _ in library.calls if n == "she_" + call.replace("_append", "")]


def test_tangents_of_what_a_call_writes_into(ctx):
    a = arguments()
    pair = [torch.zeros(3, 2, 8, dtype=torch.bfloat16), torch.zeros(3, 1, 8, dtype=torch.bfloat16)]
    with forward.dual_level():
        for i in (0, 1):
            out = list(pair)
            out[i] = forward.make_dual(out[i], torch.ones_like(out[i]))
            with pytest.raises(she.SheError, match="tangent"):
                ctx.qk_rotate(**a["qk_rotate"], out=tuple(out))
        tokens, probs = torch.zeros(2, dtype=torch.int32), forward.make_dual(torch.zeros(2), torch.ones(2))
        with pytest.raises(she.SheError, match="tangent"):
            ctx.sample(**a["sample"], out=(tokens, probs))
        sums = dict(a["sample"], logits=torch.zeros(2, 9, dtype=torch.int32), step=forward.make_dual(torch.ones(9), torch.ones(9)))
        with pytest.raises(she.SheError, match="tangent"):
            ctx.sample(**sums)
        sums = dict(a["adapters"], base=torch.zeros(3, 24, dtype=torch.int32), step=forward.make_dual(torch.ones(24), torch.ones(24)))
        with pytest.raises(she.SheError, match="tangent"):
            ctx.adapters(**sums)


@pytest.mark.parametrize("call", sorted(TENSORS))
def test_calls_without_a_tangent_are_made(library, ctx, call):  # noqa: F811
    """At a level of forward mode too, and inside a function that has a derivative of its own."""
    a = arguments()[call]
    made = "she_" + call.replace("_append", "")
    with forward.dual_level():
        getattr(ctx, call)(**a)
        assert len([n for n, _ in library.calls if n == made]) == 1
        duals = {n: forward.make_dual(a[n], torch.ones_like(a[n])) for n in names(call, a)}
        with forward._set_fwd_grad_enabled(False):
            getattr(ctx, call)(**dict(a, **duals))
        assert len([n for n, _ in library.calls if n == made]) == 2


def test_a_pair_of_results_may_be_one_tensor(library, ctx):  # noqa: F811
    a = arguments()["qk_rotate"]
    a["k"] = a["q"]
    q, k = ctx.qk_rotate(**a, out=torch.zeros(2, 3, 2, 8, dtype=torch.bfloat16))
    assert q.shape == k.shape == (3, 2, 8) and [n for n, _ in library.calls if n == "she_qk_rotate"]
