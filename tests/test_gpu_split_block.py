"""The example of a decoder's attention block in split inference: every step against its definition."""
import numpy as np
import pytest
import torch

import clear_forms as F
import paper_1906_00148_amd as she
from examples import split_block as B

pytestmark = pytest.mark.gpu


def test_split_block():
    with she.Context(she.TOY, 3, 1 << 16) as ctx:
        for option in (she.OPT_FOLD_CONSTANTS, she.OPT_GATE3_CELLS, she.OPT_COLUMN_ADDER):
            ctx.set_option(option, 1)
        r = B.step(ctx)
        assert ctx.clear_bad_ids() == 0
    dtype = torch.bfloat16
    assert np.array_equal(r["sums"], r["plain_sums"]) and r["sums"].any()
    F.check(r["qkv"], *F.adapters(**{k: r[k] for k in ("x", "down", "up", "starts", "which", "scale", "base", "step")}), dtype)
    widths = [B.Q_HEADS * B.HEAD, B.KV_HEADS * B.HEAD, B.KV_HEADS * B.HEAD]
    q, k, v = (t.unflatten(1, (-1, B.HEAD)) for t in r["qkv"].split(widths, 1))
    place = torch.from_numpy(r["place"])
    F.check(r["turned"], *F.rotate(q, r["wq"], r["cos"], r["sin"], place, B.EPS, False), dtype)
    k_pages, v_pages = (t.flatten(0, 1) for t in (r["k_pages"], r["v_pages"]))
    F.check(k_pages[r["slot"]], *F.rotate(k, r["wk"], r["cos"], r["sin"], place, B.EPS, False), dtype)
    assert torch.equal(v_pages[r["slot"]], v)
    others = np.setdiff1d(np.arange(k_pages.shape[0]), r["slot"])
    for now, before in zip((k_pages, v_pages), r["before"]):
        assert torch.equal(now[others], before.flatten(0, 1)[others])
    table, lengths = torch.tensor(r["table"], dtype=torch.int32), torch.tensor(r["lengths"], dtype=torch.int32)
    F.check(r["out"], *F.attend(r["turned"], r["k_pages"], r["v_pages"], table, r["starts"].cpu(), lengths, B.HEAD ** -0.5), dtype)
