"""What a step of generation needs around its block, by definition (include/she_clear.h), on the CPU."""
from bisect import bisect_left, bisect_right
from itertools import accumulate

import numpy as np
import torch

import clear_forms as C

F32 = 2.0 ** -24
LAST = 2 ** 31 - 1


def plan(cached, news, table, free, taken, tokens, pages, page_size, before=None):
    """(starts, lengths, positions, slots, taken, table, tokens without a place), place by place"""
    table, at = [list(row) for row in table], min(max(taken, 0), len(free))
    starts, lengths, positions, slots, lost = [0], [], [], [], 0
    for r, (c, n) in enumerate(zip(cached, news)):
        c, n = max(c, 0), min(max(n, 0), tokens - starts[-1])
        have = -(-c // page_size)
        for u in range(c, c + n):
            column = u // page_size
            slot = -1
            if column < len(table[r]):
                if column >= have and u % page_size == 0:
                    table[r][column] = -1
                    if at < len(free):
                        table[r][column] = free[at] if 0 <= free[at] < pages else -1
                        at += 1
                if 0 <= table[r][column] < pages:
                    slot = table[r][column] * page_size + u % page_size
            lost += slot < 0
            slots.append(slot)
            positions.append(min(max(before[r], 0) + u if before else u, LAST))
        starts.append(starts[-1] + n)
        lengths.append(min(c + n, LAST))
    idle = tokens - starts[-1]
    return starts, lengths, positions + [0] * idle, slots + [-1] * idle, at, table, lost


def sample_row(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, its probability) of one row of numbers; the settings are numbers of 32 bits.  Weights are in 64 bits, their sums and
    the borders exact, since a border may fall on a token (equal logits and top_p = 0.5)."""
    x = np.array(logits, np.float64)
    x[np.isnan(x)] = -np.inf
    top = x.max()
    if top == -np.inf:
        return -1, 0.0
    if not temperature > 0:
        return int(x.argmax()), 1.0
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        w = np.where(x == top, 1.0, np.where((x == -np.inf) | (top == np.inf), 0.0, np.exp((x - top) / temperature)))
    order = np.argsort(-x, kind="stable")

    def running(ids):
        return list(accumulate(map(int, np.ldexp(w[ids], 110).tolist())))
    if 0 < top_k < len(x):
        order = order[:top_k]
    if top_p < 1:
        run = running(order)
        a, b = max(top_p, 0.0).as_integer_ratio()
        order = order[:1 + bisect_left(run, -(-a * run[-1] // b), hi=len(run) - 1)]
    if min_p > 0:
        order = order[w[order] >= min(min_p, 1.0)]
    kept = np.sort(order)
    run = running(kept)
    a, b = (min(max(u, 0.0), 1 - 2.0 ** -24) if u == u else 0.0).as_integer_ratio()
    at = bisect_right(run, a * run[-1] // b)
    return int(kept[at]), w[kept[at]] / (run[-1] / 2 ** 110)


def sample(logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None, step=None):
    """(tokens, probs, the bound of the probs): a whole weight is off by 2^-44 of the largest for each token, and the result is rounded."""
    x = logits.detach().cpu()
    x = x.double().numpy() if step is None else (x.double() * step.cpu().double()).float().double().numpy()
    rows, vocab = x.shape
    settings = [[d] * rows if v is None else v.cpu().tolist() for v, d in ((temperature, 1.0), (top_k, 0), (top_p, 1.0), (min_p, 0.0))]
    got = [sample_row(x[r], float(uniform[r]), *(v[r] for v in settings)) for r in range(rows)]
    probs = torch.tensor([p for _, p in got], dtype=torch.float64)
    return torch.tensor([t for t, _ in got], dtype=torch.int32), probs, probs * (F32 + 2.0 ** -50 + vocab * 2.0 ** -44) + 2.0 ** -149


def shared(q, k_pages, v_pages, table, starts, lengths, prefix_table, prefix_requests, prefix_lengths, scale, window=0):
    """(out, bound), with the bound of clear_forms.attend.  Only what a token attends to is looked at."""
    dtype = q.dtype
    T, Hq, D = q.shape
    pages, size, Hkv = k_pages.shape[:3]
    q, k_pages, v_pages = C.cpu(q), C.cpu(k_pages), C.cpu(v_pages)
    starts, lengths, ranges, prefixes = (t.tolist() for t in (starts, lengths, prefix_requests, prefix_lengths))
    table, prefix_table = table.tolist(), prefix_table.tolist()
    out, bound = torch.zeros(T, Hq, D, dtype=torch.float64), torch.zeros(T, Hq, D, dtype=torch.float64)

    def there(row, count):
        return [(u, row[u // size], u % size) for u in range(min(count, len(row) * size)) if 0 <= row[u // size] < pages]
    for r, length in enumerate(lengths):
        b, e = starts[r], starts[r + 1]
        if e <= b:
            continue
        g = next((g for g in range(len(prefixes)) if ranges[g] <= r < ranges[g + 1]), None)
        P = 0 if g is None else max(prefixes[g], 0)
        found = ([] if g is None else there(prefix_table[g], P)) + [(P + u, page, slot) for u, page, slot in there(table[r], length)]
        place, page, slot = (torch.tensor([f[i] for f in found], dtype=torch.long) for i in range(3))
        k, v = k_pages[page, slot], v_pages[page, slot]                                # [places, Hkv, D]
        p = torch.arange(length - (e - b), length)
        seen = (place <= P + p[:, None]) & (p >= 0)[:, None]
        if window:
            seen &= place > P + p[:, None] - window
        # all tokens at once, or one by one where a place that others attend to is not finite, nor is its product with a weight of 0
        whole = bool(torch.isfinite(k).all() and torch.isfinite(v).all())
        for rows in [slice(0, e - b)] if whole else [slice(i, i + 1) for i in range(e - b)]:
            mine = seen[rows].any(0)
            if not mine.any():
                continue
            km, vm = (t[mine].repeat_interleave(Hq // Hkv, 1).transpose(0, 1).contiguous() for t in (k, v))        # [Hq, n, D]
            qm, sees = q[b:e][rows].transpose(0, 1), seen[rows][:, mine]                # [Hq, tokens, D], [tokens, n]
            some = sees.any(1)[:, None]
            s = (scale * (qm @ km.mT)).masked_fill(~sees, -np.inf)
            w = torch.where(some, torch.softmax(s, -1), 0.0)
            out[b:e][rows] = (w @ vm).transpose(0, 1)
            most = (abs(scale) * (qm.abs() @ km.abs().mT)).masked_fill(~sees, 0.0).amax(-1)
            ds = (D + 8) * F32 * most + 4 * F32 * s.masked_fill(~sees, 0.0).abs().amax(-1)
            unit = C.UNIT[dtype] + 2 * ds + (2 * sees.sum(1) + 32) * F32               # [Hq, tokens]
            limit = unit[..., None] * (w @ vm.abs())
            if dtype is torch.float16:
                limit = limit + 2.0 ** -25 * (sees.double() @ vm.abs())
            bound[b:e][rows] = limit.transpose(0, 1)
    return out, bound
