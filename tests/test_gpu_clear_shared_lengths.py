"""Attention behind shared prefixes where lengths in device memory are longer than any table reaches, up to the largest number of 32 bits: every walk
that the host chooses gives what the definition does (include/she_clear.h)."""
import pytest
import torch

from test_gpu_clear_shared import compare, ctx, inputs  # noqa: F401
from test_gpu_clear_shared_walks import CALLS

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
LAST = 2 ** 31 - 1


@pytest.mark.parametrize("name", CALLS)
def test_lengths_beyond_the_tables(ctx, name):  # noqa: F811
    _, heads, page, groups, before, after = CALLS[name]
    a = inputs(BF16, groups, *heads, page, before, after)
    # nothing is in the way where a place that is beyond a length is attended to now
    for cache in ("k_pages", "v_pages"):
        a[cache] = torch.nan_to_num(a[cache], nan=0.25)
    first = len(before)
    for prefix, own in ((None, LAST), (None, LAST - 37), (LAST, None), (LAST, LAST)):
        b = dict(a, lengths=a["lengths"].clone(), prefix_lengths=a["prefix_lengths"].clone())
        if own is not None:
            b["lengths"][first], b["lengths"][-1] = own, 1 << 30
        if prefix is not None:
            b["prefix_lengths"][0] = prefix
        for window in (0, 40, LAST - 20, LAST, 2 ** 32 - 1):
            compare(ctx, b, BF16, window, (name, prefix, own, window))
