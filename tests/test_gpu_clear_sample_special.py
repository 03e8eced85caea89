"""The choice of the next token from rows of more than 8192 logits, which several workgroups share: masks that leave little or nothing, the types' lowest
and largest values, infinities and NaN, and numbers at the ends of their range, against the definition in 64 bits (include/she_clear.h)."""
import math

import pytest
import torch

from test_gpu_clear_sample import BF16, F16, F32, INF, NAN, compare, ctx, numbers  # noqa: F401

pytestmark = pytest.mark.gpu
VOCABS = [8200, 20000]


def special_rows(vocab, dtype):
    """Twelve kinds of rows, and five whose first tiles hold nothing."""
    x, _, g = numbers(17, vocab, dtype)
    info = torch.finfo(dtype)
    x[0] = -INF
    x[1] = NAN
    x[2], x[2, vocab - 1234] = -INF, -80.0
    x[3, torch.randperm(vocab, generator=g)[:vocab - 100]] = -INF
    x[4, 5::7] = NAN
    x[5, [17, 4000, vocab - 1]] = INF
    x[6] = info.min
    x[7], x[7, 7077] = info.min, info.max
    x[8] = info.max
    x[9, ::2] = info.min
    x[10], x[10, vocab - 2] = NAN, INF
    x[11] = torch.where(torch.arange(vocab) % 2 == 0, info.tiny, -info.tiny)
    x[12, :6000] = x[12, 6010:] = info.min
    x[13, :6000] = x[13, 6010:] = -1e4
    x[14], x[14, 7000] = 0, INF
    x[15], x[15, [600, 7900]] = info.min, 3.0
    x[16, 512:] = info.min
    return x


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("vocab", VOCABS)
def test_without_filters(ctx, dtype, vocab):  # noqa: F811
    x = special_rows(vocab, dtype)
    for u in (0.0, 0.37, 0.99):
        u = torch.full((17,), u)
        compare(ctx, x, u)
        for T in (0.0, NAN, 1e-45, 1e9, INF):
            compare(ctx, x, u, temperature=torch.full((17,), T))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("filters", ["k", "p", "min", "all", "idle"])
def test_filters(ctx, dtype, vocab, filters):  # noqa: F811
    x = special_rows(vocab, dtype)
    a = {"k": dict(top_k=torch.full((17,), 60, dtype=torch.int32)), "p": dict(top_p=torch.full((17,), 0.6)), "min": dict(min_p=torch.full((17,), 0.3)),
         "all": dict(top_k=torch.full((17,), 5000, dtype=torch.int32), top_p=torch.full((17,), 0.6), min_p=torch.full((17,), 2.0)),
         "idle": dict(top_p=torch.ones(17), min_p=torch.zeros(17))}[filters]
    for u in (0.0, 0.37, 0.99):
        u = torch.full((17,), u)
        compare(ctx, x, u, **a)
        for T in (0.0, 1e-38, INF) if filters != "idle" else ():
            compare(ctx, x, u, temperature=torch.full((17,), T), **a)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_a_border_between_equal_logits_around_tiles_without_weight(ctx, dtype):  # noqa: F811
    """Half of two equal weights is the first one exactly: the token is the second, and none of those between."""
    low = [torch.finfo(dtype).min, -1e4, -100.0, -INF]
    x = torch.stack([torch.full((9216,), v) for v in low]).to(dtype)
    x[:, [600, 7900]] = 10.0
    for a in ({}, dict(min_p=torch.zeros(4)), dict(top_p=torch.full((4,), 1.0)), dict(top_k=torch.full((4,), 2, dtype=torch.int32))):
        tokens, probs = compare(ctx, x, torch.full((4,), 0.5), **a)
        assert tokens.tolist() == [7900] * 4 and probs.tolist() == [0.5] * 4
        # by definition the masked tokens of -100 have some weight, if less than any that is held
        rest = [r for r, v in enumerate(low) if v != -100.0]
        tokens, _ = compare(ctx, x[rest], torch.zeros(3), **{k: v[:3] for k, v in a.items()})
        assert tokens.tolist() == [600] * 3
        tokens, _ = ctx.sample(x.cuda(), torch.zeros(4, device="cuda"), **{k: v.cuda() for k, v in a.items()})
        assert tokens.tolist() == [600] * 4


@pytest.mark.parametrize("vocab", VOCABS)
def test_settings_at_their_ends(ctx, vocab):  # noqa: F811
    x, _, g = numbers(8, vocab, F32)
    u = torch.tensor([0.0, 1.0, 2.0, -1.0, NAN, INF, 1 - 2.0 ** -24, 2.0 ** -149])
    compare(ctx, x, u)
    compare(ctx, x, u, top_p=torch.tensor([NAN, INF, -INF, -1.0, 1.0, 0.0, 1 - 2.0 ** -24, 2.0 ** -149]))
    compare(ctx, x, u, min_p=torch.tensor([NAN, INF, -INF, -1.0, 1.0, 0.0, 1 - 2.0 ** -24, 2.0 ** -149]))
    compare(ctx, x, u, top_k=torch.tensor([0, -1, -2 ** 31, 2 ** 31 - 1, vocab, vocab - 1, 1, 2], dtype=torch.int32))


@pytest.mark.parametrize("u", [0.0, 2.0 ** -46, 2.0 ** -42, 2.0 ** -39])
def test_the_probability_of_a_token_of_hardly_any_weight(ctx, u):  # noqa: F811
    """Among tiles of logits 44 octaves below the largest, where sums of tokens have weight that each has not: the token that is drawn gets its own share."""
    octaves = torch.full((9216,), -60.0)
    octaves[9000] = 0
    octaves[0:2048:2], octaves[1:2048:2] = -44.6, -45.5
    octaves[[511, 1023, 1535, 2047]] = -44.4
    x = (octaves * math.log(2))[None]
    share = torch.softmax(x[0].double(), 0)
    token, prob = (t.item() for t in ctx.sample(x.cuda(), torch.tensor([u]).cuda()))
    # 2^-24 for the result, and the whole weight's error
    assert token < 2048 and abs(prob / share[token].item() - 1) <= 2.0 ** -24 + 9216 * 2.0 ** -44


@pytest.mark.parametrize("vocab", [100, 5000, 9000, 20000])
@pytest.mark.parametrize("setting", ["uniform", "temperature", "top_p", "min_p"])
def test_answers_in_place_of_settings(ctx, vocab, setting):  # noqa: F811
    """Rows that take the likeliest token answer early, and others' threads still look at their own settings."""
    rows = 300
    x, _, g = numbers(rows, vocab, BF16)
    a = dict(uniform=torch.rand(rows, generator=g), temperature=torch.tensor([0.0, 1.0, 0.7] * 100), top_k=torch.tensor([0, 40, 3000, 0] * 75, dtype=torch.int32),
             top_p=torch.tensor([1.0, 0.9] * 150), min_p=torch.tensor([0.0, 0.01, 0.2, 0.0] * 75))
    for names in (("uniform", "temperature"), ("uniform", "temperature", "top_k", "top_p", "min_p"), ("uniform", "temperature", "min_p")):
        if setting not in names:
            continue
        on = {k: a[k].cuda() for k in names}
        want = ctx.sample(x.cuda(), **on)
        tokens = on.get("top_k", torch.empty(rows, dtype=torch.int32, device="cuda"))
        got = ctx.sample(x.cuda(), **on, out=(tokens, on[setting]))
        assert all(torch.equal(g, w) for g, w in zip(got, want))
