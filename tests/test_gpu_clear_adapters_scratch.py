"""Gradients of a few adapters among many that no request uses: right, and without scratch for those."""
import pytest
import torch

import clear_forms as F
import paper_1906_00148_amd as she
from test_gpu_clear_adapters import inputs

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("lengths,which", [([3300, 2049, 40, 3300, 200, 2200], [250, 3, 4, 7, 250, 6]), ([2048, 2049, 2050, 31, 4100], [0, 1, 2, 3, 4]),
                                           ([100] * 60 + [3000], [5, 250] * 30 + [299])])
def test_sums_of_several_adapters_that_are_shared_out(dtype, lengths, which):
    """Adapters of more tokens than a workgroup sums (64 tiles of 32 here) beside others, in any order of their numbers."""
    starts = [0]
    for n in lengths:
        starts.append(starts[-1] + n)
    a = inputs(dtype, starts, which, 300, 20, 40, 72)
    dy = torch.randn(starts[-1], 72, generator=torch.Generator().manual_seed(9)).to(dtype).cuda()
    with she.Context(she.TOY, 18, 64) as ctx:
        for got, (want, bound), name in zip(ctx.adapters_grad(dy, **a), F.adapters_grad(dy, **a), ("dx", "ddown", "dup")):
            F.check(got, want, bound, dtype, name)


def test_scratch_is_for_the_tokens_and_not_for_all_adapters():
    """2000 adapters of rank 16 between widths of 1024, three of them in use over 6000 tokens: a place for the sums of each of them all
    would be 260 MB.  There are 190 tiles, so six places (0.8 MB), and the hidden values take 1 MB."""
    a = inputs(BF16, [0, 3000, 3010, 6000], [1999, 3, 7], 2000, 16, 1024, 1024)
    dy = torch.randn(6000, 1024, device="cuda").to(BF16)
    with she.Context(she.TOY, 18, 64) as ctx:
        torch.cuda.synchronize()
        free, reserved = torch.cuda.mem_get_info()[0], torch.cuda.memory_reserved()
        ctx.adapters_grad(dy, **a)
        torch.cuda.synchronize()
        taken = free - torch.cuda.mem_get_info()[0] - (torch.cuda.memory_reserved() - reserved)
    assert taken <= 32 << 20, taken
