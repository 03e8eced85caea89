"""The next token from a last projection that was evaluated on ciphertexts: its decrypted sums are the logits, as int32 with a step for each token."""
import numpy as np
import pytest
import torch

import paper_1906_00148_amd as she
from examples import split_block as B
from test_gpu_clear_sample import compare

pytestmark = pytest.mark.gpu


def test_the_sums_that_a_projection_decrypts_to():
    rng = np.random.default_rng(5)
    tokens, vocab = 4, 61
    with she.Context(she.TOY, 3, 1 << 16) as ctx:
        for option in (she.OPT_FOLD_CONSTANTS, she.OPT_GATE3_CELLS, she.OPT_COLUMN_ADDER):
            ctx.set_option(option, 1)
        u = rng.integers(0, 256, (tokens, B.WIDTH))
        w_sign, w_exp = rng.choice(np.array([-1, 1], np.int8), (vocab, B.WIDTH)), -rng.integers(1, 6, (vocab, B.WIDTH)).astype(np.int8)
        sums = B.encrypted_projection(ctx, u, w_sign, w_exp, 13)
        shift = -w_exp.astype(np.int64)
        assert np.array_equal(sums, ((u[:, None] >> shift) * w_sign).sum(-1) - (w_sign * (128 >> shift)).sum(-1)) and len(np.unique(sums)) > 100
        logits, step = torch.from_numpy(sums), torch.full((vocab,), 1 / 64) * (1 + torch.arange(vocab) % 3)
        uniform = torch.tensor([0.1, 0.5, 0.9, 0.3])
        compare(ctx, logits, uniform, step=step)
        got, _ = compare(ctx, logits, uniform, step=step, temperature=torch.tensor([1.0, 0.7, 2.0, 0.0]), top_k=torch.tensor([0, 9, 30, 5], dtype=torch.int32),
                         top_p=torch.tensor([0.9, 0.8, 1.0, 0.5]), min_p=torch.tensor([0.0, 0.01, 0.05, 0.0]))
        assert got[3].item() == int((logits[3] * step).argmax())
