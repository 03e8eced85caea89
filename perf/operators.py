"""The operators that run in the clear beside the encrypted layers, as cases for timing.

A client of split inference has the shared projections evaluated on ciphertexts and runs the rest of a block itself, between a
decryption and the next encryption: its adapters beside the projection's sums, the norms and the rotation of queries and keys on
their way into a paged cache, and the attention of new tokens over that cache.
"""
from __future__ import annotations

import functools
import random

import torch

own = False
DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


def listed():
    return [
        # one token of one request beside a projection as wide as the ring degree: nothing but latency
        {"name": "adapt_token", "kind": "adapt", "type": "bf16", "tokens": 1, "requests": 1, "adapters": 3, "rank": 8,
         "inputs": 1024, "outputs": 1024, "base": "same"},
        # a step of many requests, a token each, on the sums that the encrypted projection decrypts to
        {"name": "adapt_requests_96", "kind": "adapt", "type": "bf16", "tokens": 96, "requests": 96, "adapters": 40, "rank": 16,
         "inputs": 4096, "outputs": 4096, "base": "sums"},
        # ragged prompts through the widest projection of a block, with adapters of high rank
        {"name": "adapt_prompts", "kind": "adapt", "type": "f16", "tokens": 4099, "requests": 7, "adapters": 5, "rank": 64,
         "inputs": 4096, "outputs": 6144, "base": "sums"},
        # a small training step of a few requests' adapters, on a layer of the benchmark's 576 inputs
        {"name": "adapt_grad_513", "kind": "adapt_grad", "type": "f16", "tokens": 513, "requests": 6, "adapters": 3, "rank": 8,
         "inputs": 576, "outputs": 1024, "base": "none"},
        # a training step of ordinary size
        {"name": "adapt_grad_8192", "kind": "adapt_grad", "type": "bf16", "tokens": 8192, "requests": 9, "adapters": 5, "rank": 32,
         "inputs": 4096, "outputs": 4096, "base": "none"},
        # a step of a few requests: the new keys and values go into their pages
        {"name": "rotate_append_33", "kind": "rotate_append", "type": "bf16", "tokens": 33, "q_heads": 32, "kv_heads": 8, "head": 128,
         "rot": 128, "interleaved": False, "page": 16},
        # a long prompt with heads of 80 of which 40 are rotated, in pairs of neighbours
        {"name": "rotate_prompt", "kind": "rotate", "type": "f16", "tokens": 16383, "q_heads": 32, "kv_heads": 32, "head": 80,
         "rot": 40, "interleaved": True, "page": 0},
        # a training step: gradients of queries, keys and both norms' weights
        {"name": "rotate_grad", "kind": "rotate_grad", "type": "bf16", "tokens": 8192, "q_heads": 32, "kv_heads": 8, "head": 128,
         "rot": 128, "interleaved": False, "page": 0},
        # one token of a short conversation: latency
        {"name": "attend_token", "kind": "attend", "type": "bf16", "requests": 1, "new": 1, "cached": 197, "q_heads": 8, "kv_heads": 2,
         "head": 64, "page": 16, "window": 0},
        # a step of many requests of very different lengths, a token each
        {"name": "attend_tokens_64", "kind": "attend", "type": "bf16", "requests": 64, "new": 1, "cached": 16384, "q_heads": 32,
         "kv_heads": 8, "head": 128, "page": 64, "window": 0},
        # a chunk of a long prompt, the rest of which is in the cache
        {"name": "attend_chunk", "kind": "attend", "type": "bf16", "requests": 1, "new": 2048, "cached": 32768, "q_heads": 32,
         "kv_heads": 8, "head": 128, "page": 64, "window": 0},
        # a step that mixes single tokens with chunks, over a sliding window, in small pages
        {"name": "attend_mixed", "kind": "attend", "type": "f16", "requests": 24, "new": 700, "cached": 6001, "q_heads": 16,
         "kv_heads": 16, "head": 64, "page": 16, "window": 1024},
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["adapt", "adapt", "adapt_grad", "rotate_append", "rotate", "rotate_grad", "attend", "attend", "attend", "attend"])
    case = {"kind": kind, "type": rng.choice(sorted(TYPES))}
    if kind.startswith("adapt"):
        grad = kind == "adapt_grad"
        tokens = _log_int(rng, 1, 8192 if grad else 4099)
        odd = rng.random() < 0.2                                  # widths that no vector load divides
        inputs, outputs = (_log_int(rng, 64, 4096) // 8 * 8 + (rng.randint(1, 7) if odd else 0) for _ in range(2))
        requests = _log_int(rng, 1, min(tokens, 96))
        case.update(tokens=tokens, requests=requests, adapters=_log_int(rng, 1, 40 if not grad else 6), rank=_log_int(rng, 1, 32 if grad else 64),
                    inputs=inputs, outputs=outputs, base="none" if grad else rng.choice(["sums", "same", "none"]))
    elif kind.startswith("rotate"):
        append = kind == "rotate_append"
        head = 8 * rng.randint(4, 16) if rng.random() < 0.5 else rng.choice([64, 128, 256])
        kv_heads = rng.choice([1, 2, 4, 8])
        case.update(tokens=_log_int(rng, 1, 2000 if append else 4000), q_heads=kv_heads * rng.choice([1, 2, 3, 4, 8]), kv_heads=kv_heads,
                    head=head, rot=rng.choice([head, head // 2 // 2 * 2, 16]), interleaved=rng.random() < 0.4,
                    page=rng.choice([1, 16, 24, 64]) if append else 0)
    else:
        kv_heads, head = rng.choice([1, 2, 4, 8]), rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256])
        requests = _log_int(rng, 1, 64)
        new = 1 if rng.random() < 0.5 else _log_int(rng, 2, 700)
        # the plain form lays all requests out as long as the longest: no more of it than of the largest listed case
        cached = _log_int(rng, new, max(new + 1, min(16384, 400000 // requests)))
        case.update(requests=requests, new=new, cached=cached, q_heads=kv_heads * rng.choice([1, 2, 4, 7]), kv_heads=kv_heads, head=head,
                    page=rng.choice([1, 16, 24, 64, 128]), window=rng.choice([0, 0, 1, 128, 1000]))
    return case


def _layout(case):
    """What a scheduler decides, from the case alone: segments of tokens, adapters and their ranks; new tokens and lengths."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    if case["kind"].startswith("adapt"):
        T, R = case["tokens"], case["requests"]
        starts = [0] + sorted(rng.sample(range(1, T), R - 1)) + [T]
        which = [rng.randrange(case["adapters"]) if rng.random() < 0.9 else -1 for _ in range(R)]
        ranks = [rng.randint(max(1, case["rank"] // 4), case["rank"]) for _ in range(case["adapters"])]
        return starts, which, ranks
    R, new, cached = case["requests"], case["new"], case["cached"]
    if R == 1:
        return [0, new], [cached], None
    news = [1 if rng.random() < 0.5 else rng.randint(1, new) for _ in range(R)]
    lengths = [rng.randint(n, max(n, cached)) for n in news]
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    return starts, lengths, None


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEVICE)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    dtype = TYPES[case["type"]]

    def normal(*shape, std=1.0, as_type=dtype):
        return (torch.randn(*shape, generator=gen, device=DEVICE) * std).to(as_type)

    kind, state = case["kind"], {"case": case}
    if kind.startswith("adapt"):
        T, A, r, K, N = (case[k] for k in ("tokens", "adapters", "rank", "inputs", "outputs"))
        starts, which, ranks = _layout(case)
        state.update(x=normal(T, K), down=normal(A, r, K, std=K ** -0.5), up=normal(A, r, N, std=0.3 * r ** -0.5), starts=_ints(starts),
                     which=_ints(which), ranks=_ints(ranks), scale=torch.rand(A, generator=gen, device=DEVICE) * 2 + 0.25, base=None, step=None)
        if kind == "adapt_grad":
            state["dy"] = normal(T, N)
        elif case["base"] == "same":
            state["base"] = normal(T, N)
        elif case["base"] == "sums":                              # 16-bit accumulators, as decrypted, and their outputs' steps
            state["base"] = torch.randint(-8192, 8192, (T, N), generator=gen, device=DEVICE, dtype=torch.int32)
            state["step"] = (torch.rand(N, generator=gen, device=DEVICE) + 0.5) / 4096
        return state
    if kind.startswith("rotate"):
        T, Hq, Hkv, D, rot = (case[k] for k in ("tokens", "q_heads", "kv_heads", "head", "rot"))
        qkv = normal(T, (Hq + 2 * Hkv) * D)                       # one projection's output: the heads are views of it
        q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([Hq * D, Hkv * D, Hkv * D], 1))
        places = 2 * T + 77
        angle = torch.arange(places, device=DEVICE)[:, None] * 10000.0 ** (-torch.arange(rot // 2, device=DEVICE) * 2.0 / rot)
        state.update(q=q, k=k, v=v, wq=normal(D, std=0.2, as_type=torch.float32) + 1, wk=normal(D, std=0.2, as_type=torch.float32) + 1,
                     cos=angle.cos(), sin=angle.sin(), positions=torch.randint(0, places, (T,), generator=gen, device=DEVICE, dtype=torch.int32))
        if kind == "rotate_grad":
            state.update(dq=normal(T, Hq, D), dk=normal(T, Hkv, D))
        elif kind == "rotate_append":
            pages = T // case["page"] + 9
            state.update(k_pages=normal(pages, case["page"], Hkv, D), v_pages=normal(pages, case["page"], Hkv, D),
                         slots=torch.randperm(pages * case["page"], generator=gen, device=DEVICE)[:T])
        return state
    Hq, Hkv, D, page = (case[k] for k in ("q_heads", "kv_heads", "head", "page"))
    starts, lengths, _ = _layout(case)
    width = max(-(-n // page) for n in lengths)
    total = sum(-(-n // page) for n in lengths) + 5
    order = torch.randperm(total, generator=gen, device=DEVICE, dtype=torch.int32)
    row = _ints([[p if p * page < n else -1 for p in range(width)] for n in lengths])
    before = _ints([0] + [-(-n // page) for n in lengths[:-1]]).cumsum(0)
    table = torch.where(row >= 0, order[(row.clamp(min=0) + before[:, None]).long()], row)
    state.update(q=normal(starts[-1], Hq, D), k_pages=normal(total, page, Hkv, D), v_pages=normal(total, page, Hkv, D), table=table,
                 starts=_ints(starts), lengths=_ints(lengths), scale=D ** -0.5, most_new=max(b - a for a, b in zip(starts, starts[1:])),
                 most_cached=max(lengths))
    return state


# ---- the framework's calls
@functools.lru_cache(None)
def _context():
    """The context that a client has anyway; the operators use its stream and its scratch."""
    import paper_1906_00148_amd as she
    return she.Context(she.TOY, 1, 64)


def _run_own(s):
    ctx, case = _context(), s["case"]
    kind = case["kind"]
    if kind == "adapt":
        return ctx.adapters(s["x"], s["down"], s["up"], s["starts"], s["which"], s["scale"], ranks=s["ranks"], base=s["base"], step=s["step"])
    if kind == "adapt_grad":
        return ctx.adapters_grad(s["dy"], s["x"], s["down"], s["up"], s["starts"], s["which"], s["scale"], ranks=s["ranks"])
    if kind == "rotate":
        return ctx.qk_rotate(s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], s["positions"], eps=EPS, interleaved=case["interleaved"])
    if kind == "rotate_append":
        q = ctx.qk_rotate_append(s["q"], s["k"], s["v"], s["wq"], s["wk"], s["cos"], s["sin"], s["positions"], s["k_pages"], s["v_pages"],
                                 s["slots"], eps=EPS, interleaved=case["interleaved"])
        return q, s["k_pages"], s["v_pages"]
    if kind == "rotate_grad":
        return ctx.qk_rotate_grad(s["dq"], s["dk"], s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], s["positions"], eps=EPS,
                                  interleaved=case["interleaved"])
    return ctx.attend_pages(s["q"], s["k_pages"], s["v_pages"], s["table"], s["starts"], s["lengths"], s["scale"], window=case["window"])


# ---- the plain forms
def _columns(s):
    """[tokens, adapters * rank]: the scale of the token's adapter in the columns that this adapter's rank has, else 0"""
    A, r = s["down"].shape[:2]
    token = torch.arange(s["x"].shape[0], device=DEVICE)
    adapter = s["which"][torch.searchsorted(s["starts"], token, right=True) - 1]
    used = torch.arange(r, device=DEVICE) < s["ranks"][:, None]
    mine = adapter[:, None] == torch.arange(A, device=DEVICE)
    return ((mine * s["scale"])[:, :, None] * used).flatten(1)


def _adapt(s):
    columns = _columns(s)
    y = (s["x"].float() @ s["down"].float().flatten(0, 1).T * columns) @ s["up"].float().flatten(0, 1)
    if s["base"] is not None:
        y = y + (s["base"].float() if s["step"] is None else s["base"].float() * s["step"])
    return y.to(s["x"].dtype)


def _adapt_grad(s):
    columns, x, dy = _columns(s), s["x"].float(), s["dy"].float()
    down, up = s["down"].float().flatten(0, 1), s["up"].float().flatten(0, 1)
    g, h = dy @ up.T * columns, x @ down.T * columns
    dtype = s["x"].dtype
    return (g @ down).to(dtype), (g.T @ x).to(dtype).view_as(s["down"]), (h.T @ dy).to(dtype).view_as(s["up"])


def _pairs(x, rot, interleaved):
    x = x[..., :rot]
    return (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:])


def _turn(x, s, backwards=False):
    rot, interleaved = s["case"]["rot"], s["case"]["interleaved"]
    at = s["positions"].long()
    cos, sin = s["cos"][at][:, None], s["sin"][at][:, None]
    sin = -sin if backwards else sin
    a, b = _pairs(x, rot, interleaved)
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _rotate(x, w, s):
    x32 = x.float()
    return _turn(x32 * torch.rsqrt(x32.square().mean(-1, keepdim=True) + EPS) * w, s).to(x.dtype)


def _rotate_grad(dy, x, w, s):
    x32, g = x.float(), _turn(dy.float(), s, backwards=True)
    r = torch.rsqrt(x32.square().mean(-1, keepdim=True) + EPS)
    dx = r * (w * g) - x32 * r.pow(3) * (w * g * x32).mean(-1, keepdim=True)
    return dx.to(x.dtype), (g * x32 * r).sum((0, 1))


def _attend(s):
    case = s["case"]
    Hq, Hkv, page = case["q_heads"], case["kv_heads"], case["page"]
    starts, lengths = s["starts"].long(), s["lengths"].long()
    news = starts[1:] - starts[:-1]
    new, place = torch.arange(s["most_new"], device=DEVICE), torch.arange(s["most_cached"], device=DEVICE)
    at = s["table"].long()[:, place // page].clamp(min=0) * page + place % page
    k, v = (t.flatten(0, 1)[at].float().transpose(1, 2) for t in (s["k_pages"], s["v_pages"]))      # [requests, kv heads, places, head]
    live = new < news[:, None]
    token = torch.where(live, starts[:-1, None] + new, 0)
    q = s["q"][token].float().unflatten(2, (Hkv, Hq // Hkv)).permute(0, 2, 3, 1, 4)                # [requests, kv heads, group, new, head]
    reach = (lengths - news)[:, None] + new                                                       # the last place that a token sees
    seen = (place <= reach[..., None]) & (place < lengths[:, None, None])
    if case["window"]:
        seen &= place > reach[..., None] - case["window"]
    R, G, n = q.shape[0], q.shape[2], q.shape[3]
    score = ((q.flatten(2, 3) @ k.transpose(2, 3)).unflatten(2, (G, n)) * s["scale"]).masked_fill(~seen[:, None, None], float("-inf"))
    top = score.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = (score - top).exp()
    o = (p.flatten(2, 3) @ v).unflatten(2, (G, n)) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    o = o.permute(0, 3, 1, 2, 4).flatten(2, 3)                                                    # [requests, new, heads, head]
    return o[live].to(s["q"].dtype)


def run(state):
    if own:
        return _run_own(state)
    s, kind = state, state["case"]["kind"]
    if kind == "adapt":
        return _adapt(s)
    if kind == "adapt_grad":
        return _adapt_grad(s)
    if kind == "rotate":
        return _rotate(s["q"], s["wq"], s), _rotate(s["k"], s["wk"], s)
    if kind == "rotate_append":
        s["k_pages"].flatten(0, 1)[s["slots"]] = _rotate(s["k"], s["wk"], s)
        s["v_pages"].flatten(0, 1)[s["slots"]] = s["v"]
        return _rotate(s["q"], s["wq"], s), s["k_pages"], s["v_pages"]
    if kind == "rotate_grad":
        (dq, dwq), (dk, dwk) = _rotate_grad(s["dq"], s["q"], s["wq"], s), _rotate_grad(s["dk"], s["k"], s["wk"], s)
        return dq, dk, dwq, dwk
    return _attend(s)


# ---- what a pass cannot do without
def work(case):
    kind = case["kind"]
    if kind.startswith("adapt"):
        T, K, N = case["tokens"], case["inputs"], case["outputs"]
        starts, which, ranks = _layout(case)
        weights = 2 * (K + N) * sum(ranks[a] for a in set(which) if a >= 0)
        # multiplications and additions of the two (or, for the gradients, six) products of each token with its adapter's rank
        products = 2 * (K + N) * sum((b - a) * ranks[w] for a, b, w in zip(starts, starts[1:], which) if w >= 0)
        if kind == "adapt_grad":
            out = 2 * (K + N) * case["adapters"] * case["rank"]
            return {"bytes": T * (2 * K + 2 * N + 2 * K) + weights + out, "flops": 2 * products + products * K // (K + N)}
        base = {"none": 0, "same": 2, "sums": 4}[case["base"]]
        return {"bytes": T * (2 * K + (2 + base) * N) + weights, "flops": products}
    if kind.startswith("rotate"):
        T, Hq, Hkv, D, rot = (case[k] for k in ("tokens", "q_heads", "kv_heads", "head", "rot"))
        heads = T * (Hq + Hkv) * D
        table = T * 4 * (rot + 1)
        if kind == "rotate_grad":
            return {"bytes": 6 * heads + table, "flops": 16 * heads}
        extra = T * (4 * Hkv * D + 8) if kind == "rotate_append" else 0
        return {"bytes": 4 * heads + table + extra, "flops": 8 * heads}
    starts, lengths, _ = _layout(case)
    window, D = case["window"], case["head"]
    pairs = places = 0
    for a, b, length in zip(starts, starts[1:], lengths):
        first = length - (b - a)                                  # the first new token's place
        seen = [min(p + 1, window) if window else p + 1 for p in range(first, length)]
        pairs += sum(seen)
        places += length - (first + 1 - seen[0])
    return {"bytes": 4 * starts[-1] * case["q_heads"] * D + 4 * places * case["kv_heads"] * D, "flops": 4 * D * case["q_heads"] * pairs}


# ---- the definitions in 64 bits, token by token or request by request
def _exact_adapt(s, starts, which, ranks):
    x, down, up = s["x"].double(), s["down"].double(), s["up"].double()
    T, N = x.shape[0], up.shape[2]
    y = torch.zeros(T, N, dtype=torch.float64, device=DEVICE)
    if s["base"] is not None:
        y += s["base"].double() * (1.0 if s["step"] is None else s["step"].double())
    for a, b, w in zip(starts, starts[1:], which):
        if w >= 0:
            r = ranks[w]
            y[a:b] += s["scale"][w].double() * ((x[a:b] @ down[w, :r].mT) @ up[w, :r])
    return y


def _exact_adapt_grad(s, starts, which, ranks):
    x, dy, down, up = s["x"].double(), s["dy"].double(), s["down"].double(), s["up"].double()
    dx, ddown, dup = torch.zeros_like(x), torch.zeros_like(down), torch.zeros_like(up)
    for a, b, w in zip(starts, starts[1:], which):
        if w >= 0:
            r, scale = ranks[w], s["scale"][w].double()
            h, g = scale * (x[a:b] @ down[w, :r].mT), scale * (dy[a:b] @ up[w, :r].mT)
            dx[a:b] = g @ down[w, :r]
            ddown[w, :r] += g.mT @ x[a:b]
            dup[w, :r] += h.mT @ dy[a:b]
    return dx, ddown, dup


def _exact_places(case):
    """indexes of the first and the second member of every pair"""
    half = torch.arange(case["rot"] // 2, device=DEVICE)
    return (2 * half, 2 * half + 1) if case["interleaved"] else (half, half + case["rot"] // 2)


def _exact_rotate(x, w, s):
    x = x.double()
    n = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w.double()
    first, second = _exact_places(s["case"])
    cos, sin = s["cos"].double()[s["positions"].long()].unsqueeze(1), s["sin"].double()[s["positions"].long()].unsqueeze(1)
    y = n.clone()
    y[..., first] = n[..., first] * cos - n[..., second] * sin
    y[..., second] = n[..., first] * sin + n[..., second] * cos
    return y


def _exact_rotate_grad(dy, x, w, s):
    x, dy, w = x.double(), dy.double(), w.double()
    first, second = _exact_places(s["case"])
    cos, sin = s["cos"].double()[s["positions"].long()].unsqueeze(1), s["sin"].double()[s["positions"].long()].unsqueeze(1)
    g = dy.clone()
    g[..., first] = dy[..., first] * cos + dy[..., second] * sin
    g[..., second] = dy[..., second] * cos - dy[..., first] * sin
    root = (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt()
    unit = x / root
    dx = (w * g - unit * (w * g * unit).sum(-1, keepdim=True) / x.shape[-1]) / root
    return dx, (g * unit).sum(0).sum(0)


def _exact_attend(s, starts, lengths):
    case = s["case"]
    G, page = case["q_heads"] // case["kv_heads"], case["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    for request, (a, b, length) in enumerate(zip(starts, starts[1:], lengths)):
        where = s["table"][request, :-(-length // page)].long()
        k, v = (t[where].flatten(0, 1)[:length] for t in (s["k_pages"], s["v_pages"]))
        place = torch.arange(length, device=DEVICE)
        last = torch.arange(length - (b - a), length, device=DEVICE)[:, None]
        hidden = (place > last) | (place <= last - case["window"] if case["window"] else place < 0)
        for head in range(case["q_heads"]):
            score = s["scale"] * (s["q"][a:b, head].double() @ k[:, head // G].double().T)
            out[a:b, head] = score.masked_fill(hidden, float("-inf")).softmax(-1) @ v[:, head // G].double()
    return out


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "adapt":
        return _exact_adapt(s, *_layout(case))
    if kind == "adapt_grad":
        return _exact_adapt_grad(s, *_layout(case))
    if kind == "rotate":
        return _exact_rotate(s["q"], s["wq"], s), _exact_rotate(s["k"], s["wk"], s)
    if kind == "rotate_append":
        k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
        k_pages.flatten(0, 1)[s["slots"]] = _exact_rotate(s["k"], s["wk"], s)
        v_pages.flatten(0, 1)[s["slots"]] = s["v"].double()
        return _exact_rotate(s["q"], s["wq"], s), k_pages, v_pages
    if kind == "rotate_grad":
        (dq, dwq), (dk, dwk) = _exact_rotate_grad(s["dq"], s["q"], s["wq"], s), _exact_rotate_grad(s["dk"], s["k"], s["wk"], s)
        return dq, dk, dwq, dwk
    return _exact_attend(s, *_layout(case)[:2])
