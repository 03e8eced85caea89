"""The rest of a generation step in the clear, as cases for timing.

Beside the adapters, norms and attention of perf/operators.py, a client's step needs its places in the cache worked out from the
requests' lengths (plan), the attention of requests that begin with the same long text (shared), and the choice of the next token
from the last projection's logits (sample).
"""
from __future__ import annotations

import functools
import random

import torch

own = False
DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # the next token of one conversation: nothing but latency
        {"name": "plan_token", "kind": "plan", "requests": 1, "new": 1, "cached": 197, "page": 16, "width": 64, "spare": 0},
        # a step of many requests, most with one token, in a batch padded to a fixed size
        {"name": "plan_step_509", "kind": "plan", "requests": 509, "new": 3, "cached": 16384, "page": 16, "width": 1100, "spare": 37},
        # a night's queue of ragged prompts
        {"name": "plan_prompts", "kind": "plan", "requests": 2500, "new": 400, "cached": 3000, "page": 64, "width": 64, "spare": 0},
        # two answers drawn from one short prompt: latency
        {"name": "shared_pair", "kind": "shared", "type": "bf16", "prefixes": 1, "requests": 2, "new": 1, "prefix": 333, "own": 41,
         "q_heads": 8, "kv_heads": 2, "head": 64, "page": 16, "window": 0},
        # a step of 64 requests of a token each behind one long document
        {"name": "shared_tokens_64", "kind": "shared", "type": "bf16", "prefixes": 1, "requests": 64, "new": 1, "prefix": 32768, "own": 500,
         "q_heads": 32, "kv_heads": 8, "head": 128, "page": 64, "window": 0},
        # several documents, each with the requests that ask about it, a few drafted tokens each
        {"name": "shared_documents_5", "kind": "shared", "type": "f16", "prefixes": 5, "requests": 97, "new": 4, "prefix": 9001, "own": 700,
         "q_heads": 16, "kv_heads": 16, "head": 64, "page": 16, "window": 0},
        # questions of up to 300 tokens about one text, read for the first time
        {"name": "shared_questions", "kind": "shared", "type": "bf16", "prefixes": 1, "requests": 24, "new": 300, "prefix": 8192, "own": 300,
         "q_heads": 32, "kv_heads": 8, "head": 128, "page": 64, "window": 0},
        # a layer with a sliding window that reaches back into the shared text, odd heads
        {"name": "shared_window", "kind": "shared", "type": "f16", "prefixes": 2, "requests": 33, "new": 2, "prefix": 5000, "own": 900,
         "q_heads": 28, "kv_heads": 4, "head": 80, "page": 24, "window": 4096},
        # the next token of one conversation
        {"name": "sample_one", "kind": "sample", "type": "bf16", "rows": 1, "vocab": 32001, "filters": "p"},
        # a small batch whose logits are the sums that the encrypted projection decrypts to
        {"name": "sample_sums_13", "kind": "sample", "type": "sums", "rows": 13, "vocab": 50021, "filters": "all"},
        # a step of 64 requests without any filter
        {"name": "sample_plain_64", "kind": "sample", "type": "f16", "rows": 64, "vocab": 100000, "filters": "none"},
        # a large batch over a large vocabulary, every request with settings of its own
        {"name": "sample_batch_256", "kind": "sample", "type": "f32", "rows": 256, "vocab": 131072, "filters": "all"},
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["plan", "shared", "shared", "shared", "sample", "sample"])
    case = {"kind": kind}
    if kind == "plan":
        page = rng.choice([1, 16, 24, 64, 128])
        requests = _log_int(rng, 1, 2500)
        new = 1 if rng.random() < 0.5 else _log_int(rng, 2, 400)
        cached = _log_int(rng, 1, min(16384, 500000 * page // requests))
        case.update(requests=requests, new=new, cached=cached, page=page, width=(cached + new) // page + rng.randint(1, 64),
                    spare=rng.choice([0, 1, 50]))
    elif kind == "shared":
        kv_heads, head = rng.choice([1, 2, 4, 8]), rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256])
        requests = _log_int(rng, 1, 96)
        new = 1 if rng.random() < 0.5 else _log_int(rng, 2, 200)
        prefix = _log_int(rng, 16, max(17, min(32768, 12000000 // (requests * new))))
        case.update(type=rng.choice(["bf16", "f16"]), prefixes=rng.randint(1, min(6, requests)), requests=requests, new=new, prefix=prefix,
                    own=_log_int(rng, new, max(new + 1, min(2000, 100000 // requests))), q_heads=kv_heads * rng.choice([1, 2, 4, 7]),
                    kv_heads=kv_heads, head=head, page=rng.choice([1, 16, 24, 64, 128]), window=rng.choice([0, 0, 0, 100, 3000]))
    else:
        case.update(type=rng.choice(["bf16", "f16", "f32", "sums"]), rows=_log_int(rng, 1, 256), vocab=_log_int(rng, 100, 131072),
                    filters=rng.choice(["none", "k", "p", "min", "all", "all"]))
    return case


def _layout(case):
    """What the requests ask for, from the case alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    R, new = case["requests"], case["new"]
    if case["kind"] == "plan":
        if R == 1:
            return [case["cached"]], [new]
        # some requests pause for a step
        news = [0 if rng.random() < 0.05 else 1 if rng.random() < 0.5 else rng.randint(1, new) for _ in range(R)]
        return [0 if rng.random() < 0.1 else rng.randint(0, case["cached"]) for _ in range(R)], news
    G = case["prefixes"]
    ranges = [0] + sorted(rng.sample(range(1, R), G - 1)) + [R]
    prefixes = [case["prefix"]] + [rng.randint(max(1, case["prefix"] // 4), case["prefix"]) for _ in range(G - 1)]
    news = [new if R <= 2 else rng.randint(1, new) for _ in range(R)]
    lengths = [case["own"] if R <= 2 else rng.randint(n, max(n, case["own"])) for n in news]
    return ranges, prefixes, news, lengths


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEVICE)


def _sums(values):
    total = [0]
    for v in values:
        total.append(total[-1] + v)
    return total


def _prepare_plan(case, gen):
    R, page, width = case["requests"], case["page"], case["width"]
    cached, news = (_ints(v) for v in _layout(case))
    order = torch.randperm(R, generator=gen, device=DEVICE)
    cached, news = cached[order], news[order]
    have = (cached + page - 1) // page
    # pages in no order: those that the requests have, then the free ones, some of which are taken already
    held, taken = int(have.sum()), 11
    need = int(((cached + news + page - 1) // page).sum()) - held
    ids = torch.randperm(held + taken + need + 50, generator=gen, device=DEVICE, dtype=torch.int32)
    column = torch.arange(width, device=DEVICE)
    first = have.cumsum(0) - have
    table = torch.where(column < have[:, None], ids[(first[:, None] + column).clamp(max=held - 1 if held else 0)], -1).contiguous()
    return {"cached": cached, "news": news, "table": table, "free": ids[held:].contiguous(), "taken": _ints([taken]),
            "before": torch.randint(0, 5000, (R,), generator=gen, device=DEVICE, dtype=torch.int32),
            "tokens": int(news.sum()) + case["spare"], "pages": ids.numel()}


def _tables(counts, page, ids):
    """A row of page ids for each of these numbers of places, -1 beyond them; takes the ids from the front."""
    need = [-(-n // page) for n in counts]
    column = torch.arange(max(1, *need) if need else 1, device=DEVICE)
    first = _ints(_sums(need)[:-1], torch.int64)
    held = column < _ints(need)[:, None]
    return torch.where(held, ids[torch.where(held, first[:, None] + column, 0)], -1), sum(need)


def _prepare_shared(case, gen):
    Hq, Hkv, D, page = (case[k] for k in ("q_heads", "kv_heads", "head", "page"))
    dtype = TYPES[case["type"]]
    ranges, prefixes, news, lengths = _layout(case)
    total = sum(-(-n // page) for n in prefixes + lengths) + 5
    ids = torch.randperm(total, generator=gen, device=DEVICE, dtype=torch.int32)
    prefix_table, used = _tables(prefixes, page, ids)
    table, _ = _tables(lengths, page, ids[used:])
    starts = _sums(news)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE).to(dtype)
    return {"q": normal(starts[-1], Hq, D), "k_pages": normal(total, page, Hkv, D), "v_pages": normal(total, page, Hkv, D), "table": table,
            "starts": _ints(starts), "lengths": _ints(lengths), "prefix_table": prefix_table, "prefix_requests": _ints(ranges),
            "prefix_lengths": _ints(prefixes), "scale": D ** -0.5,
            # the scheduler's own copies, which the plain form pads by
            "groups": [(a, b, starts[a], starts[b], p, max(news[a:b]), max(lengths[a:b])) for a, b, p in zip(ranges, ranges[1:], prefixes)]}


def _prepare_sample(case, gen):
    rows, vocab, filters = case["rows"], case["vocab"], case["filters"]
    logits = torch.randn(rows, vocab, generator=gen, device=DEVICE) * 2
    # a few likely tokens, in some rows one that has nearly all of the mass, and in every fourth row a grammar that rules out most tokens
    likely = torch.randint(0, vocab, (rows, 1), generator=gen, device=DEVICE)
    likely = (likely + torch.arange(20, device=DEVICE) * (vocab // 20)) % vocab
    logits.scatter_(1, likely, torch.randn(rows, 20, generator=gen, device=DEVICE) * 2 + 9)
    logits[::3, vocab // 2] += 12
    state = {"step": None}
    if case["type"] == "sums":
        state["step"] = (torch.rand(vocab, generator=gen, device=DEVICE) + 0.5) / 256
        state["logits"] = (logits * 256).round().to(torch.int32)
    else:
        ruled_out = torch.rand(rows, vocab, generator=gen, device=DEVICE) < 0.7
        ruled_out &= (torch.arange(rows, device=DEVICE) % 4 == 1)[:, None]
        state["logits"] = logits.masked_fill_(ruled_out, float("-inf")).to(TYPES[case["type"]])

    def per_row(low, high, off, share=0.3):
        """a setting for every row, `off` in some"""
        v = torch.rand(rows, generator=gen, device=DEVICE) * (high - low) + low
        return torch.where(torch.rand(rows, generator=gen, device=DEVICE) < share, off, v)
    state["uniform"] = torch.rand(rows, generator=gen, device=DEVICE)
    state["temperature"] = per_row(0.5, 1.3, 1.0)
    if filters == "all" and rows > 8:
        state["temperature"][::8] = 0.0                           # some requests want the likeliest token
    state["top_k"] = per_row(1, 200, 0.0).to(torch.int32) if filters in ("k", "all") else None
    state["top_p"] = per_row(0.5, 0.99, 1.0) if filters in ("p", "all") else None
    state["min_p"] = per_row(0.01, 0.2, 0.0) if filters in ("min", "all") else None
    return state


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    make = {"plan": _prepare_plan, "shared": _prepare_shared, "sample": _prepare_sample}[case["kind"]]
    return dict(make(case, gen), case=case)


# ---- the framework's calls
@functools.lru_cache(None)
def _context():
    """The context that a client has anyway; the operators use its stream and its scratch."""
    import paper_1906_00148_amd as she
    return she.Context(she.TOY, 1, 64)


def _run_own(s):
    ctx, case = _context(), s["case"]
    if case["kind"] == "plan":
        return (*ctx.plan_pages(s["cached"], s["news"], s["table"], s["free"], s["taken"], s["tokens"], s["pages"], case["page"],
                                before=s["before"]), s["table"])
    if case["kind"] == "shared":
        return ctx.attend_shared(s["q"], s["k_pages"], s["v_pages"], s["table"], s["starts"], s["lengths"], s["prefix_table"],
                                 s["prefix_requests"], s["prefix_lengths"], s["scale"], window=case["window"])
    return ctx.sample(s["logits"], s["uniform"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                      step=s["step"])


# ---- the plain forms
def _plan(s):
    page, tokens, free, table = s["case"]["page"], s["tokens"], s["free"], s["table"]
    width = table.shape[1]
    cached, news = s["cached"].long(), s["news"].long()
    starts = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEVICE), news.cumsum(0).clamp(max=tokens)])
    lengths = cached + starts[1:] - starts[:-1]
    have, need = ((n + page - 1) // page for n in (cached, lengths))
    fresh = need.clamp(max=width) - have.clamp(max=width)
    first = s["taken"].long() + fresh.cumsum(0) - fresh
    column = torch.arange(width, device=DEVICE)
    at = first[:, None] + column - have[:, None]
    new = (column >= have[:, None]) & (column < need[:, None])
    page_id = torch.where(at < free.numel(), free[at.clamp(0, free.numel() - 1)], -1)
    table.copy_(torch.where(new, page_id, table))
    token = torch.arange(tokens, device=DEVICE)
    request = torch.searchsorted(starts[1:], token, right=True).clamp(max=cached.numel() - 1)
    live = token < starts[-1]
    place = cached[request] + token - starts[request]
    mine = table[request, (place // page).clamp(max=width - 1)].long()
    slots = torch.where(live & (place // page < width) & (mine >= 0), mine * page + place % page, -1)
    positions = torch.where(live, s["before"][request] + place, 0)
    taken = (s["taken"] + fresh.sum()).clamp(max=free.numel())
    return starts.int(), lengths.int(), positions.int(), slots, taken.int(), table


def _shared(s):
    case = s["case"]
    Hkv, G, D, page = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["head"], case["page"]
    keys, values = s["k_pages"].flatten(0, 1), s["v_pages"].flatten(0, 1)
    out = torch.empty_like(s["q"])

    def places(table, count):
        """where the first `count` places of each row lie"""
        place = torch.arange(count, device=DEVICE)
        return table.long()[:, place // page].clamp(min=0) * page + place % page
    for g, (a, b, first, last, prefix, new, longest) in enumerate(s["groups"]):
        starts, lengths = s["starts"][a:b + 1].long(), s["lengths"][a:b].long()
        news, R = starts[1:] - starts[:-1], b - a
        step = torch.arange(new, device=DEVICE)
        live = step < news[:, None]
        q = s["q"][torch.where(live, starts[:-1, None] + step, first)].float().unflatten(2, (Hkv, G)).permute(2, 0, 3, 1, 4)   # [Hkv, R, G, new, D]
        at = places(s["prefix_table"][g:g + 1], prefix)[0]
        pk, pv = (t[at].float().transpose(0, 1) for t in (keys, values))                             # [Hkv, prefix, D]
        at = places(s["table"][a:b], longest)
        ok, ov = (t[at].float().permute(2, 0, 1, 3) for t in (keys, values))                         # [Hkv, R, longest, D]
        behind = (q.reshape(Hkv, -1, D) @ pk.transpose(1, 2).contiguous()).unflatten(1, (R, G, new))
        mine = (q.flatten(2, 3) @ ok.transpose(2, 3).contiguous()).unflatten(2, (G, new))
        reach = (lengths - news)[:, None] + step                                                     # a token's own place
        place = torch.arange(longest, device=DEVICE)
        seen = (place <= reach[..., None]) & (place < lengths[:, None, None])
        score = torch.cat([behind, mine.masked_fill(~seen[:, None], float("-inf"))], -1) * s["scale"]
        if case["window"]:
            place = torch.arange(prefix + longest, device=DEVICE)
            score.masked_fill_((place <= prefix + reach[..., None] - case["window"])[:, None], float("-inf"))
        p = (score - score.amax(-1, keepdim=True)).exp()
        total = p.sum(-1, keepdim=True)
        o = (p[..., :prefix].reshape(Hkv, -1, prefix) @ pv).unflatten(1, (R, G, new))
        o = (o + (p[..., prefix:].flatten(2, 3) @ ov).unflatten(2, (G, new))) / total
        o = o.permute(1, 3, 0, 2, 4).flatten(2, 3)                                                   # [R, new, heads, D]
        out[first:last] = o[live].to(out.dtype)
    return out


def _sample(s):
    logits, rows = s["logits"], s["logits"].shape[0]
    # in 64 bits: sums of many small terms, and a border that they are next to
    x = logits.double() if s["step"] is None else (logits.double() * s["step"].double()).float().double()
    top = x.amax(-1, keepdim=True)
    greedy = s["temperature"] <= 0
    w = ((x - top) / torch.where(greedy, 1.0, s["temperature"]).double()[:, None]).exp()
    likeliest = x.argmax(-1)
    if s["top_k"] is not None or s["top_p"] is not None:
        order = x.sort(dim=-1, descending=True, stable=True).indices
        sorted_w = w.gather(-1, order)
        if s["top_k"] is not None:
            k = torch.where(s["top_k"] > 0, s["top_k"], x.shape[1])
            sorted_w = sorted_w * (torch.arange(x.shape[1], device=DEVICE) < k[:, None])
        if s["top_p"] is not None:
            run = sorted_w.cumsum(-1)
            p = s["top_p"].double()[:, None]
            sorted_w = sorted_w * ((run - sorted_w < p * run[:, -1:]) | (p >= 1))
        w = torch.zeros_like(w).scatter_(-1, order, sorted_w)
    if s["min_p"] is not None:
        w = w * (w >= s["min_p"].double()[:, None])
    run = w.cumsum(-1)
    token = (run <= s["uniform"].double()[:, None] * run[:, -1:]).sum(-1)
    token = torch.where(greedy, likeliest, token)
    prob = torch.where(greedy, 1.0, w[torch.arange(rows, device=DEVICE), token] / run[:, -1])
    return token.int(), prob.float()


def run(state):
    if own:
        return _run_own(state)
    return {"plan": _plan, "shared": _shared, "sample": _sample}[state["case"]["kind"]](state)


# ---- what a pass cannot do without
def work(case):
    kind = case["kind"]
    if kind == "plan":
        page, (cached, news) = case["page"], _layout(case)
        fresh = sum(-(-(c + n) // page) - -(-c // page) for c, n in zip(cached, news))
        tokens = sum(news)
        # lengths, numbers and offsets in; starts, lengths and, for each token, position and slot out; an id for each new page
        return {"bytes": 12 * len(news) + 8 * len(news) + 12 * (tokens + case["spare"]) + 8 * fresh, "flops": 4 * tokens + 8 * len(news)}
    if kind == "shared":
        ranges, prefixes, news, lengths = _layout(case)
        D, window = case["head"], case["window"]
        places = pairs = 0
        for a, b, prefix in zip(ranges, ranges[1:], prefixes):
            lowest = prefix
            for n, length in zip(news[a:b], lengths[a:b]):
                at = [prefix + length - n + i for i in range(n)]
                seen = [min(p + 1, window) if window else p + 1 for p in at]
                pairs += sum(seen)
                lowest = min(lowest, at[0] + 1 - seen[0])
                places += at[-1] + 1 - max(prefix, at[0] + 1 - seen[0])
            places += prefix - lowest
        return {"bytes": 4 * sum(news) * case["q_heads"] * D + 4 * places * case["kv_heads"] * D, "flops": 4 * D * case["q_heads"] * pairs}
    rows, vocab = case["rows"], case["vocab"]
    each = 2 if case["type"] in ("bf16", "f16") else 4
    step = 4 * vocab if case["type"] == "sums" else 0
    # a weight for each logit, and its sum
    return {"bytes": rows * (each * vocab + 28) + step, "flops": 4 * rows * vocab}


# ---- the definitions, request by request or row by row
def _exact_plan(s):
    case = s["case"]
    page = case["page"]
    cached, news, free, table, before = (s[k].tolist() for k in ("cached", "news", "free", "table", "before"))
    starts, lengths, positions, slots, at = [0], [], [], [], int(s["taken"])
    for r, (c, n) in enumerate(zip(cached, news)):
        for place in range(c, c + n):
            column = place // page
            if place % page == 0 and column < case["width"]:      # the first place of a page
                table[r][column] = free[at]
                at += 1
            slots.append(table[r][column] * page + place % page if column < case["width"] else -1)
            positions.append(before[r] + place)
        starts.append(starts[-1] + n)
        lengths.append(c + n)
    idle = s["tokens"] - len(slots)
    return (_ints(starts), _ints(lengths), _ints(positions + [0] * idle), _ints(slots + [-1] * idle, torch.int64), _ints([at]), _ints(table))


def _exact_shared(s):
    case = s["case"]
    group, page, window = case["q_heads"] // case["kv_heads"], case["page"], case["window"]
    ranges, prefixes, news, lengths = _layout(case)
    starts = _sums(news)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)

    def pages(row, count):
        return [t[row[:-(-count // page)].long()].flatten(0, 1)[:count] for t in (s["k_pages"], s["v_pages"])]
    for g, prefix in enumerate(prefixes):
        shared = pages(s["prefix_table"][g], prefix)
        for r in range(ranges[g], ranges[g + 1]):
            k, v = (torch.cat(t) for t in zip(shared, pages(s["table"][r], lengths[r])))
            all_places = prefix + lengths[r]
            place = torch.arange(all_places, device=DEVICE)
            last = torch.arange(all_places - news[r], all_places, device=DEVICE)[:, None]
            hidden = (place > last) | (place <= last - window if window else place < 0)
            for head in range(case["q_heads"]):
                score = s["scale"] * (s["q"][starts[r]:starts[r + 1], head].double() @ k[:, head // group].double().T)
                out[starts[r]:starts[r + 1], head] = score.masked_fill(hidden, float("-inf")).softmax(-1) @ v[:, head // group].double()
    return out


def _exact_sample(s):
    tokens, probs = [], []
    logits = s["logits"].double()
    if s["step"] is not None:
        logits = (logits * s["step"].double()).float().double()   # a logit is a number of 32 bits
    settings = [None if s[k] is None else s[k].tolist() for k in ("temperature", "top_k", "top_p", "min_p", "uniform")]
    for r, row in enumerate(logits):
        temperature, k, p, least, u = (None if v is None else v[r] for v in settings)
        if temperature <= 0:
            tokens.append(int((row == row.max()).nonzero()[0]))
            probs.append(1.0)
            continue
        mass = torch.softmax(row / temperature, 0)
        ids = torch.argsort(-row, stable=True)
        if k is not None and 0 < k < len(ids):
            ids = ids[:k]
        if p is not None and p < 1:
            head = mass[ids].cumsum(0)
            ids = ids[:1 + int((head < p * head[-1]).sum())]
        if least is not None and least > 0:
            ids = ids[mass[ids] >= least * mass.max()]
        ids = ids.sort().values
        run = mass[ids].cumsum(0)
        at = ids[int(torch.searchsorted(run, u * run[-1], right=True))]
        tokens.append(int(at))
        probs.append(float(mass[at] / run[-1]))
    return _ints(tokens), _ints(probs, torch.float64)


def exact(case, seed):
    return {"plan": _exact_plan, "shared": _exact_shared, "sample": _exact_sample}[case["kind"]](prepare(case, seed))
