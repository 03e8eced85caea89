"""Attention over a paged cache where a call has many rows: the kernel for tiles of them, at masks, tables and sizes where it can go wrong,
against the definition in 64 bits."""
import pytest
import torch

import clear_forms as F
import paper_1906_00148_amd as she
from test_gpu_clear_attend import compare, inputs

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    with she.Context(she.TOY, 15, 64) as c:
        yield c


# tokens and lengths of each request, heads, page, the table's columns, window
BEYOND_THE_TABLE = [([2048], [2048], 1, 1, 64, 16, 17, 0), ([300], [2000], 4, 1, 128, 16, 65, 0), ([500, 1, 300], [1100, 1500, 400], 4, 2, 64, 24, 43, 0),
                    ([600, 200], [900, 700], 2, 1, 96, 1, 777, 700), ([400], [1300], 4, 1, 256, 16, 67, 0)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("news,lengths,Hq,Hkv,D,page,width,window", BEYOND_THE_TABLE)
def test_lengths_beyond_the_table(ctx, dtype, news, lengths, Hq, Hkv, D, page, width, window):
    """Places that the table has no column for are attended to by nobody, wherever in a step of the kernel they begin."""
    a = inputs(dtype, news, lengths, Hq, Hkv, D, page)
    a["table"] = a["table"][:, :width]
    compare(ctx, a, dtype, window)
