"""The attention block of a decoder in split inference, for a step of several requests.

The projection to queries, keys and values belongs to a server, which sees ciphertexts only: its weights are powers of two and it is
evaluated bit by bit (shift-accumulate, Section 3.2 of arXiv 1906.00148).  The rest is the client's own and runs in the clear on
the client's GPU: each request's low-rank adapter beside the projection's decrypted sums, the norms of queries and keys with the
rotation of their positions, which puts keys and values into the pages of the cache, and the attention of the new tokens over it.

    python examples/split_block.py
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1906_00148_amd as she                                # noqa: E402
from paper_1906_00148_amd import layers                           # noqa: E402

WIDTH, Q_HEADS, KV_HEADS, HEAD, RANK, PAGE, BITS = 24, 4, 2, 8, 4, 4, 8
OUTPUTS = (Q_HEADS + 2 * KV_HEADS) * HEAD
EPS = 1e-6


def encrypted_projection(ctx, u, w_sign, w_exp, acc_bits):
    """The server's part: u [tokens][WIDTH] unsigned 8-bit numbers, encrypted here; returns the sums, decrypted."""
    bits = (u[..., None] >> np.arange(BITS)) & 1
    ids = np.arange(bits.size, dtype=np.uint32).reshape(bits.shape)
    ctx.encrypt_bits(bits, 7, ids)
    chain = layers.Chain(ctx, bits.size)
    # (u - 128) w: the constant part of the sum is known to the server
    bias = -(w_sign.astype(np.int32) * (128 >> -w_exp.astype(np.int32))).sum(1)
    ctx.defer_begin()                                             # the tokens' circuits as one
    out = [chain.dense(row, w_sign, w_exp, acc_bits, bias) for row in ids]
    ctx.defer_run()
    got = ctx.decrypt(np.stack(out)).astype(np.int64)             # [tokens][OUTPUTS][acc_bits]
    value = (got << np.arange(acc_bits)).sum(-1)
    return np.where(got[..., -1] == 1, value - (1 << acc_bits), value).astype(np.int32)


def step(ctx, seed=1, dtype=torch.bfloat16):
    """One step of three requests, of one, three and two new tokens; returns its outputs and what they were made from."""
    rng = np.random.default_rng(seed)
    gen = torch.Generator().manual_seed(seed)
    cached, new = [5, 0, 9], [1, 3, 2]
    lengths, starts = [c + n for c, n in zip(cached, new)], np.concatenate([[0], np.cumsum(new)])
    T = int(starts[-1])

    def dev(values, ty=torch.int32):
        return torch.as_tensor(np.asarray(values)).to("cuda", ty)

    # the activations, as the client has them, and as it quantizes them for the server
    x = torch.randn(T, WIDTH, generator=gen).to(dtype).cuda()
    quantum = 4.0 / 128
    u = np.clip(np.rint(x.float().cpu().numpy() / quantum) + 128, 0, 255).astype(np.int64)
    w_sign, w_exp = rng.choice(np.array([-1, 1], np.int8), (OUTPUTS, WIDTH)), -rng.integers(1, 6, (OUTPUTS, WIDTH)).astype(np.int8)
    sums = encrypted_projection(ctx, u, w_sign, w_exp, 13)
    plain_sums = ((u[:, None] >> -w_exp.astype(np.int64)) * w_sign).sum(-1) - (w_sign * (128 >> -w_exp.astype(np.int64))).sum(-1)

    # the client's own weights and its cache
    s = dict(x=x, down=(torch.randn(2, RANK, WIDTH, generator=gen) / WIDTH ** 0.5).to(dtype).cuda(),
             up=(torch.randn(2, RANK, OUTPUTS, generator=gen) / RANK ** 0.5).to(dtype).cuda(), starts=dev(starts), which=dev([1, -1, 0]),
             scale=dev([0.5, 1.0], torch.float32), base=dev(sums), step=torch.full((OUTPUTS,), quantum, device="cuda"))
    wq, wk = (1 + 0.1 * torch.randn(2, HEAD, generator=gen)).cuda()
    angle = torch.arange(32)[:, None] * 100.0 ** (-torch.arange(HEAD // 2) * 2.0 / HEAD)
    cos, sin = angle.cos().cuda(), angle.sin().cuda()
    table = [[6, 2, -1], [0, -1, -1], [3, 7, 1]]
    k_pages, v_pages = torch.randn(2, 8, PAGE, KV_HEADS, HEAD, generator=gen).to(dtype).cuda()
    place = np.concatenate([np.arange(c, c + n) for c, n in zip(cached, new)])
    slot = [table[r][p // PAGE] * PAGE + p % PAGE for r, n in enumerate(new) for p in place[starts[r]:starts[r] + n]]

    before = k_pages.clone(), v_pages.clone()
    qkv = ctx.adapters(**s)
    q, k, v = (t.unflatten(1, (-1, HEAD)) for t in qkv.split([Q_HEADS * HEAD, KV_HEADS * HEAD, KV_HEADS * HEAD], 1))
    turned = ctx.qk_rotate_append(q, k, v, wq, wk, cos, sin, dev(place), k_pages, v_pages, dev(slot, torch.int64), eps=EPS)
    out = ctx.attend_pages(turned, k_pages, v_pages, dev(table), s["starts"], dev(lengths))
    return dict(s, out=out, qkv=qkv, turned=turned, sums=sums, plain_sums=plain_sums, wq=wq, wk=wk, cos=cos, sin=sin, place=place, slot=slot,
                table=table, lengths=lengths, k_pages=k_pages, v_pages=v_pages, before=before)


def main():
    with she.Context(she.TOY, 3, 1 << 16) as ctx:
        for option in (she.OPT_FOLD_CONSTANTS, she.OPT_GATE3_CELLS, she.OPT_COLUMN_ADDER):
            ctx.set_option(option, 1)
        r = step(ctx)
        exact = np.array_equal(r["sums"], r["plain_sums"])
        print(f"projection of {len(r['sums'])} tokens on ciphertexts: sums {'as' if exact else 'NOT as'} in the clear")
        print(f"attention's outputs {tuple(r['out'].shape)}, norm {float(r['out'].float().norm()):.4f}, ids out of range: {ctx.clear_bad_ids()}")
    return 0 if exact else 1


if __name__ == "__main__":
    sys.exit(main())
