"""How exact attention for single tokens is: nothing but the result's own rounding to the type shows."""
import pytest
import torch

import clear_forms as F
import paper_1906_00148_amd as she
from test_gpu_clear_attend import inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    with she.Context(she.TOY, 22, 64) as c:
        yield c


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("news,lengths,Hq,Hkv,D", [([1], [197], 8, 2, 64), ([1] * 6, [3, 64, 100, 700, 1500, 4000], 8, 2, 128), ([1], [6000], 4, 1, 128),
                                                   ([3, 2], [300, 900], 2, 1, 256), ([1, 1], [50, 350], 4, 4, 80)])
def test_weights_are_held_in_more_than_the_type(ctx, dtype, news, lengths, Hq, Hkv, D):
    """The error in the 2-norm is that of rounding the definition once, up to the 2 % that sums in 32 bits and weights in twice the type's bits
    (roundings 2^8 times smaller) may add."""
    a = inputs(dtype, news, lengths, Hq, Hkv, D, 16)
    got, want = F.cpu(ctx.attend_pages(**a)), F.attend(**a)[0]
    assert float((got - want).norm()) <= 1.02 * float((F.cpu(want.to(dtype)) - want).norm())
