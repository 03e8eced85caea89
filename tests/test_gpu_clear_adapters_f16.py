"""Adapters in float16 where numbers that are summed or handed on side by side differ by as much as the type allows: a token's result does
not depend on the tokens beside it.  Against the definition in 64 bits."""
import pytest
import torch

import clear_forms as F
import paper_1906_00148_amd as she
from test_gpu_clear_adapters import dev

pytestmark = pytest.mark.gpu
F16 = torch.float16


@pytest.fixture(scope="module")
def ctx():
    with she.Context(she.TOY, 19, 64) as c:
        yield c


def inputs(r, K, N, starts, which, A, large):
    """Tokens `large` have inputs of about 2^14, the others of 2^-14, and hidden values of 2^10 and 2^-18; results are of about these
    inputs' sizes."""
    g = torch.Generator().manual_seed(21)
    T = starts[-1]

    def normal(*shape):
        return torch.randn(*shape, generator=g)
    size = torch.full((T, 1), 2.0 ** -14)
    size[list(large)] = 2.0 ** 13
    return dict(x=(normal(T, K).clamp(-3, 3) * size).half().cuda(), down=(normal(A, r, K) / 16 * K ** -0.5).half().cuda(),
                up=(normal(A, r, N) * 16 * r ** -0.5).half().cuda(), starts=dev(starts), which=dev(which), scale=torch.tensor([1.0, 0.75, 1.5])[:A].cuda())


# rank, widths, segments, adapters; the single launch of a few tiles, two launches, ranks of several chunks, odd widths
CASES = [(8, 64, 128, [0, 5, 40], [0, 1], 2), (20, 128, 256, [0, 33, 64, 100], [2, 0, 1], 3), (64, 256, 512, [0, 700], [0], 1),
         (130, 128, 264, [0, 40, 95], [1, 0], 2), (12, 71, 133, [0, 64], [0], 1)]


@pytest.mark.parametrize("r,K,N,starts,which,A", CASES)
def test_one_large_token_among_small_ones(ctx, r, K, N, starts, which, A):
    a = inputs(r, K, N, starts, which, A, large=range(3, starts[-1], 37))
    want, bound = F.adapters(**a)
    got = ctx.adapters(**a)
    F.check(got, want, bound, F16)
    small = [t for t in range(starts[-1]) if t % 37 != 3]
    F.check(got[small], want[small], bound[small], F16)             # in the 2-norm too


@pytest.mark.parametrize("r,K,N,starts,which,A", CASES)
def test_gradients_of_a_token_do_not_depend_on_the_others(ctx, r, K, N, starts, which, A):
    """dx as the result above (the matrices have changed places); and the gradients of the matrices where the ranks differ as much, which
    are the rows of their results."""
    a = inputs(r, N, K, starts, which, A, large=range(3, starts[-1], 37))
    dy, down, up = a["x"], a["up"], a["down"]
    b = dict(a, x=torch.randn(starts[-1], K, generator=torch.Generator().manual_seed(3)).half().cuda(), down=down, up=up)
    dx, _, _ = ctx.adapters_grad(dy, **b)
    want, bound = F.adapters_grad(dy, **b)[0]
    F.check(dx, want, bound, F16)
    # ranks of about 2^12 and of 2^-16 side by side
    size = torch.where(torch.arange(r) % 5 == 2, 2.0 ** 12, 2.0 ** -16)[None, :, None]
    g = torch.Generator().manual_seed(5)
    c = dict(a, x=torch.randn(starts[-1], K, generator=g).half().cuda(), down=(torch.randn(A, r, K, generator=g) * size * K ** -0.5 / 64).half().cuda(),
             up=(torch.randn(A, r, N, generator=g) * size * N ** -0.5 / 64).half().cuda())
    c["scale"] = c["scale"] * 4
    dy = torch.randn(starts[-1], N, generator=g).half().cuda()
    for got, (want, bound), name in list(zip(ctx.adapters_grad(dy, **c), F.adapters_grad(dy, **c), ("dx", "ddown", "dup")))[1:]:
        F.check(got, want, bound, F16, name)
