"""The clear side's operators by definition, in 64 bits on the CPU, with the bounds that their rounding allows.

UNIT is the unit roundoff of a type: a result rounded once to nearest is off by at most UNIT of itself.  What comes before is held
in 32 bits, whose sums of n terms are off by at most n * 2^-24 of the sum of the terms' sizes; each bound below names its n.
"""
import numpy as np
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -24}          # f16 results below its normal range
# what is left of a number that is handed on as two of the type
SPLIT = {torch.bfloat16: 2.0 ** -16, torch.float16: 2.0 ** -21}
F32 = 2.0 ** -24


def cpu(t):
    return None if t is None else t.detach().to("cpu", torch.float64)


def check(got, want, bound, dtype, what=""):
    """Every element within UNIT of itself and `bound`; finite parts within UNIT of the whole in the 2-norm (errors that are
    independent from element to element, as roundings are, add up to less; a term that is left out does not)."""
    got, want = cpu(got), cpu(want)
    assert got.shape == want.shape
    bound = bound + UNIT.get(dtype, 0) * want.abs() + TINY.get(dtype, 0)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what
    off = (got - want).abs()[fine]
    assert bool((off <= bound[fine]).all()), (what, float((off / bound[fine].clamp(min=1e-300)).max()))
    if dtype in UNIT and off.numel():
        assert float(off.norm()) <= UNIT[dtype] * float(want[fine].norm()) + TINY[dtype] * off.numel() ** 0.5, what


# ---- adapters
def adapters(x, down, up, starts, which, scale, ranks=None, base=None, step=None, **_):
    """(out, bound)"""
    dtype = x.dtype
    x, down, up, scale = map(cpu, (x, down, up, scale))
    T, K = x.shape
    A, r, N = up.shape
    out, size = torch.zeros(T, N, dtype=torch.float64), torch.zeros(T, N, dtype=torch.float64)
    if base is not None:
        out = cpu(base) * (1.0 if step is None else cpu(step))
        size = out.abs() * 4 * F32
    for s, a in enumerate(which.tolist()):
        b, e = starts[s].item(), starts[s + 1].item()
        if e <= b or not 0 <= a < A:
            continue
        n = r if ranks is None else min(max(int(ranks[a]), 0), r)
        out[b:e] += scale[a] * (x[b:e] @ down[a, :n].T) @ up[a, :n]
        # the sums over K and the rank, the split of the hidden values, and a few single roundings
        size[b:e] += (SPLIT[dtype] + (K + r + 16) * F32) * scale[a].abs() * (x[b:e].abs() @ down[a, :n].abs().T) @ up[a, :n].abs()
    return out, size


def adapters_grad(dy, x, down, up, starts, which, scale, ranks=None, base=None, **_):
    """((dx, bound), (ddown, bound), (dup, bound))"""
    dtype = x.dtype
    dx = adapters(dy, up, down, starts, which, scale, ranks, base)       # the same form with the matrices' parts exchanged
    dy, x, down, up, scale = map(cpu, (dy, x, down, up, scale))
    A, r, K = down.shape
    N = up.shape[2]
    dd, sd, du, su = torch.zeros_like(down), torch.zeros_like(down), torch.zeros_like(up), torch.zeros_like(up)
    T = x.shape[0]
    for s, a in enumerate(which.tolist()):
        b, e = starts[s].item(), starts[s + 1].item()
        if e <= b or not 0 <= a < A:
            continue
        n = r if ranks is None else min(max(int(ranks[a]), 0), r)
        g, h = scale[a] * dy[b:e] @ up[a, :n].T, scale[a] * x[b:e] @ down[a, :n].T
        dd[a, :n] += g.T @ x[b:e]
        du[a, :n] += h.T @ dy[b:e]
        unit = SPLIT[dtype] + (max(K, N) + T + 32) * F32
        sd[a, :n] += unit * (scale[a].abs() * dy[b:e].abs() @ up[a, :n].abs().T).T @ x[b:e].abs()
        su[a, :n] += unit * (scale[a].abs() * x[b:e].abs() @ down[a, :n].abs().T).T @ dy[b:e].abs()
    return dx, (dd, sd), (du, su)


# ---- queries and keys
def _places(D, rot, interleaved):
    half = torch.arange(rot // 2)
    return (2 * half, 2 * half + 1) if interleaved else (half, half + rot // 2)


def rotate(x, w, cos, sin, positions, eps, interleaved):
    """(out, bound) of one of q and k"""
    x, cos, sin = cpu(x), cpu(cos), cpu(sin)
    D = x.shape[-1]
    w = torch.ones(D, dtype=torch.float64) if w is None else cpu(w)
    n = x / ((x * x).mean(-1, keepdim=True) + eps).sqrt() * w
    at = positions.cpu().long()
    ok = ((at >= 0) & (at < cos.shape[0]))[:, None, None]
    at = at.clamp(0, cos.shape[0] - 1)
    c, s = cos[at][:, None], sin[at][:, None]
    i, j = _places(D, 2 * cos.shape[1], interleaved)
    y, size = n.clone(), n.abs()
    y[..., i], y[..., j] = n[..., i] * c - n[..., j] * s, n[..., j] * c + n[..., i] * s
    size[..., i], size[..., j] = (n[..., i] * c).abs() + (n[..., j] * s).abs(), (n[..., j] * c).abs() + (n[..., i] * s).abs()
    # the sum over D under a root (half of it), and a dozen single roundings
    return torch.where(ok, y, 0.0), torch.where(ok, size * (D / 2 + 24) * F32, 0.0)


def rotate_grad(dy, x, w, cos, sin, positions, eps, interleaved):
    """((dx, bound), (dw, bound))"""
    x, cos, sin, dy = cpu(x), cpu(cos), cpu(sin), cpu(dy)
    D = x.shape[-1]
    w = torch.ones(D, dtype=torch.float64) if w is None else cpu(w)
    at = positions.cpu().long()
    ok = ((at >= 0) & (at < cos.shape[0]))[:, None, None]
    at = at.clamp(0, cos.shape[0] - 1)
    c, s = cos[at][:, None], sin[at][:, None]
    i, j = _places(D, 2 * cos.shape[1], interleaved)
    g, gs = dy.clone(), dy.abs()
    g[..., i], g[..., j] = dy[..., i] * c + dy[..., j] * s, dy[..., j] * c - dy[..., i] * s
    gs[..., i], gs[..., j] = (dy[..., i] * c).abs() + (dy[..., j] * s).abs(), (dy[..., j] * c).abs() + (dy[..., i] * s).abs()
    r = 1 / ((x * x).mean(-1, keepdim=True) + eps).sqrt()
    u = x * r
    dx = r * (w * g - u * (w * g * u).mean(-1, keepdim=True))
    size = r * (w.abs() * gs + u.abs() * (w.abs() * gs * u.abs()).mean(-1, keepdim=True))
    unit = (2 * D + 40) * F32
    # a weight's sum: over the steps of a wavefront, its lanes, and the workgroups' sums eight at a time
    chain = D / 2 + 24 + 256
    return ((torch.where(ok, dx, 0.0), torch.where(ok, size * unit, 0.0)),
            ((g * u * ok).sum((0, 1)), (gs * u.abs() * ok).sum((0, 1)) * chain * F32))


# ---- attention
def attend(q, k_pages, v_pages, table, starts, lengths, scale, window=0):
    """(out, bound).  Only what a token attends to is looked at."""
    dtype = q.dtype
    T, Hq, D = q.shape
    pages, size, Hkv = k_pages.shape[:3]
    q, k_pages, v_pages = cpu(q), cpu(k_pages), cpu(v_pages)
    out, bound = torch.zeros(T, Hq, D, dtype=torch.float64), torch.zeros(T, Hq, D, dtype=torch.float64)
    table = table.cpu().tolist()
    for r, length in enumerate(lengths.tolist()):
        b, e = starts[r].item(), starts[r + 1].item()
        places = [u for u in range(min(length, len(table[r]) * size)) if 0 <= table[r][u // size] < pages]
        if e <= b:
            continue
        where = torch.tensor(places, dtype=torch.long)
        page = torch.tensor([table[r][u // size] for u in places], dtype=torch.long)
        k, v = k_pages[page, where % size], v_pages[page, where % size]                # [places, Hkv, D]
        for t in range(b, e):
            p = length - (e - b) + (t - b)
            mine = where <= p
            if window:
                mine &= where > p - window
            if not mine.any():
                continue
            km = k[mine].repeat_interleave(Hq // Hkv, 1).transpose(0, 1)               # [Hq, n, D]
            vm = v[mine].repeat_interleave(Hq // Hkv, 1).transpose(0, 1)
            s = scale * (km @ q[t][:, :, None])[..., 0]
            w = torch.softmax(s, -1)
            out[t] = (w[:, None] @ vm)[:, 0]
            # a score is off by the sum over D and a few roundings of itself, and its weight by twice that; weights are rounded to the
            # type, their sum and the second product's go over all places
            ds = (D + 8) * F32 * (abs(scale) * (km.abs() @ q[t].abs()[:, :, None])[..., 0]).amax(-1) + 4 * F32 * s.abs().amax(-1)
            n = mine.sum().item()
            unit = UNIT[dtype] + 2 * ds + (2 * n + 32) * F32
            bound[t] = unit[:, None] * (w[:, None] @ vm.abs())[:, 0]
            if dtype is torch.float16:                                                 # weights below its normal range
                bound[t] += 2.0 ** -25 * vm.abs().sum(1)
    return out, bound


def pages_of(lengths, page, spare=3, seed=0):
    """A table of pages in random order for requests of these lengths, -1 beyond them, and the pages there are."""
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in lengths]
    total = sum(need) + spare
    order = rng.permutation(total)
    table = np.full((len(lengths), max(max(need), 1)), -1, np.int32)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    return torch.from_numpy(table), total
