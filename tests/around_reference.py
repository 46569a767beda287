"""The operators around K-interval attention from their definitions in 64 bits, on
the device of their inputs, with bounds on what a correct kernel may be off by.

`u` is the relative error of one rounding to the outputs' type (2^-8 for bfloat16,
2^-24 for float32), `E` that of an fp32 operation. A sum of n terms in fp32 is off by at
most n E times the sum of their magnitudes."""
import math

import torch

E = 2.0 ** -24


def unit(dtype):
    return torch.finfo(dtype).eps / 2


def seen(T, window, sinks, device, Tk=None, first=0):
    i = first + torch.arange(T, device=device)[:, None]
    j = torch.arange(T if Tk is None else Tk, device=device)
    return (j <= i) & ((i - j < window) | (j < sinks))


def window(q, k, v, win, sinks, lengths=None, dO=None):
    """{name: (value, bound)} of o, lse and, with dO, dq, dk, dv."""
    dtype = q.dtype
    B, H, T, d = q.shape
    G, u = H // k.shape[1], unit(dtype)
    low = u if dtype == torch.bfloat16 else 0.0  # rounding of computed operands
    scale = 1.0 / math.sqrt(d)
    sc = float(torch.tensor(scale, dtype=torch.float32))
    q, k, v = q.double(), k.double().repeat_interleave(G, 1), v.double().repeat_interleave(G, 1)
    see = seen(T, win, sinks, q.device).expand(B, 1, T, T)
    n = torch.full((B,), T, device=q.device) if lengths is None else lengths.clamp(0, T)
    row = torch.arange(T, device=q.device) < n[:, None]
    see = see & row[:, None, :, None] & row[:, None, None, :]
    row = row[:, None, :, None]
    # (rows past a sequence hold anything)
    q, k, v = (torch.where(row, x, 0.0) for x in (q, k, v))
    s = (q @ k.transpose(-1, -2)) * scale
    s = s.masked_fill(~see, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    empty = total == 0
    lse = top + torch.log(total)
    p = p / torch.where(empty, 1.0, total)
    o = p @ v
    # a score is off by d + 3 roundings of the sum of its terms' magnitudes, a weight by
    # that twice (its own and the row sum's), the exponential and the sum over the keys
    mag = (q.abs() @ k.abs().transpose(-1, -2)) * scale + abs(sc - scale) / scale * s.abs().nan_to_num(posinf=0)
    es = ((d + 3) * E * mag).masked_fill(~see, 0.0)
    worst = es.amax(-1, keepdim=True) + (s - top).abs().masked_fill(~see, 0.0) * 4 * E + 4 * E
    rp = 2 * worst + (T + 8) * E + low
    A = (p * rp) @ v.abs()
    bo = u * o.abs() + A + (T + 4) * E * (p @ v.abs()) + 1e-30
    bl = torch.where(empty, 0.0, worst.amax(-1, keepdim=True) + (T + 8) * E + 4 * E * (lse.abs() + top.abs())
                     .nan_to_num(posinf=0))
    out = {"o": (o, bo), "lse": (lse[..., 0], bl[..., 0])}
    if dO is None:
        return out
    g = torch.where(row, dO.double(), 0.0)
    dp = g @ v.transpose(-1, -2)
    D = (g * o).sum(-1, keepdim=True)
    ds = p * (dp - D)
    # D from an output that is off by bo; dO.v by its own sum's roundings
    edp = (d + 2) * E * (g.abs() @ v.abs().transpose(-1, -2))
    eD = (g.abs() * bo).sum(-1, keepdim=True) + (d + 2) * E * (g.abs() * o.abs()).sum(-1, keepdim=True)
    eds = p * (edp + eD) + (rp + 2 * E) * ds.abs() + low * ds.abs()
    fold = lambda x: x.reshape(B, H // G, G, T, d).sum(2)  # noqa: E731
    n_terms = (T + 4) * E
    for name, a, b, ea, r in (("dq", ds * scale, k, eds * scale, 1),
                              ("dk", ds.transpose(-1, -2) * scale, q, eds.transpose(-1, -2) * scale, G),
                              ("dv", p.transpose(-1, -2), g, (rp * p).transpose(-1, -2), G)):
        x, e = a @ b, ea @ b.abs() + G * n_terms * (a.abs() @ b.abs())
        if r > 1 or name != "dq":
            x, e = fold(x), fold(e)
        out[name] = (x, u * x.abs() + e + 1e-30)
    return out


def rotary(x, freq, layout, factor, positions, back=False):
    """The rotated tensor and its bound, in units of E times the pair's magnitudes: the
    rest of the angle rounded (1), sine and cosine to 4 units in the last place (4),
    their product with the factor (1), a product and a sum (2); and the output's
    rounding."""
    n = freq.shape[0]
    a = positions.double()[:, None, :, None] * freq
    c, s = torch.cos(a) * factor, torch.sin(a) * factor * (-1 if back else 1)
    t = x.double()
    r = t[..., :2 * n]
    x0, x1 = (r[..., :n], r[..., n:]) if layout == "half" else (r[..., 0::2], r[..., 1::2])
    y0, y1 = x0 * c - x1 * s, x1 * c + x0 * s
    size = (x0.abs() + x1.abs()) * abs(factor)
    if layout == "half":
        y, size = torch.cat((y0, y1), -1), torch.cat((size, size), -1)
    else:
        y, size = torch.stack((y0, y1), -1).flatten(-2), torch.stack((size, size), -1).flatten(-2)
    bound = unit(x.dtype) * y.abs() + 8 * E * size
    return (torch.cat((y, t[..., 2 * n:]), -1),
            torch.cat((bound, torch.zeros_like(t[..., 2 * n:])), -1))


LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def held(x):
    """What the 4-bit cache stands for once it holds x [..., d]."""
    g = x.double().reshape(*x.shape[:-1], -1, 32)
    top = g.abs().amax(-1, keepdim=True)
    bad = ~torch.isfinite(top)
    e = torch.full_like(top, -126.0)
    while True:
        more = (top > 6 * torch.exp2(e)) & (e < 125) & ~bad
        if not more.any():
            break
        e = torch.where(more, e + 1, e)
    s = torch.exp2(e)
    level = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    off = ((g.abs() / s)[..., None] - level).abs()
    best = off.amin(-1, keepdim=True)
    even = torch.arange(8, device=x.device) % 2 == 0
    tie = (off == best)
    pick = torch.where(tie & even, 2, torch.where(tie, 1, 0)).argmax(-1)
    y = torch.copysign(level[pick] * s, g)
    return torch.where(bad, math.nan, y).reshape(x.shape)


def cached_scores(q, k):
    """Scores of q [H, T, d] against the keys k [Hkv, n, d] that the cache stands for."""
    H, T, d = q.shape
    G = H // k.shape[0]
    return (q.double() @ k.double().repeat_interleave(G, 0).transpose(1, 2)) / math.sqrt(d)


def cached(q, k, v, n, K=4, calib="fwm", tau=8.0, recon="nearest", win=0, sinks=0):
    """Attention of q [H, T, d], the last of n tokens, over keys and values [Hkv, n, d];
    (value, bound). A weight within rounding of a midpoint or of the FWM cut may fall on
    the other side: the bound then has the whole step of that weight."""
    dtype = q.dtype
    H, T, d = q.shape
    G, u = H // k.shape[0], unit(dtype)
    low = u if dtype == torch.bfloat16 else 0.0
    if n == 0:
        z = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
        return z, z
    s = cached_scores(q, k)
    k, v = (x.double().repeat_interleave(G, 0) for x in (k, v))
    see = seen(T, win if win else n + T, sinks if win else 0, q.device, n, n - T).expand(H, T, n)
    top = s.masked_fill(~see, -math.inf).amax(-1, keepdim=True)
    some = top > -math.inf
    top = torch.where(some, top, 0.0)
    low_s = torch.where(some, s.masked_fill(~see, math.inf).amin(-1, keepdim=True), 0.0)
    z = s - top
    es = (d + 4) * E * (q.double().abs() @ k.abs().transpose(1, 2)) / math.sqrt(d)
    es = torch.where(see, es, 0.0).amax(-1, keepdim=True) + 4 * E * (top.abs() + low_s.abs())
    if recon == "softmax":
        w = torch.exp(z)
        ew = w * (2 * es + 8 * E * (1 + z.abs()))
    else:
        span = top - low_s if calib == "minmax" else torch.full_like(top, tau)
        flat = (calib == "minmax") & (span <= 1e-12)
        span = torch.where(flat, 1.0, span)
        h = span / K
        pos = (z + span) / h
        r = torch.floor(pos).clamp(max=K - 1)
        if calib != "resolved":
            r = r.clamp(min=0)
        t = (pos - r).clamp(0, 1)
        lo, hi = torch.exp(r * h - span), torch.exp((r + 1) * h - span)
        # positions move by the scores' errors, over the step
        ep = 4 * es / h + 16 * E * (pos.abs() + K)
        if recon == "lerp":
            w = lo + t * (hi - lo)
            # the chord's slope, at most the next interval's, and the grid's own rounding
            ew = ep * (hi - lo) * torch.exp(h) + w * (16 * E * (1 + z.abs() + span) + 2 * es)
        else:
            w = torch.where(t >= 0.5, hi, lo)
            ew = w * (16 * E * (1 + z.abs() + span) + (2 * es if calib == "minmax" else 0))
            ew = ew + torch.where((t - 0.5).abs() <= 2 * ep, hi - lo, 0.0)
        if calib == "fwm":
            w, ew = torch.where(pos < 0, 0.0, w), torch.where(pos < 0, 0.0, ew)
            ew = torch.where(pos.abs() <= ep, ew + torch.exp(-span), ew)
        w, ew = torch.where(flat, 1.0, w), torch.where(flat, 8 * E, ew)
    w, ew = torch.where(see, w, 0.0), torch.where(see, ew, 0.0)
    total = w.sum(-1, keepdim=True)
    total = torch.where(total == 0, 1.0, total)
    v = torch.where(see.any(1)[..., None], v, 0.0)
    o = (w / total) @ v
    A = (w / total) @ v.abs()
    # (the largest weight is 1, so the computed sum is at least that but for its rounding)
    least = (total - ew.sum(-1, keepdim=True)).clamp(min=0.9)
    rel = ew.sum(-1, keepdim=True) / least + 2 * (n + 16) * E
    return o, u * o.abs() + (ew / least) @ v.abs() + (rel + low) * A + 1e-30


def within(got, want, bound, what):
    got = got.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, 0.0, (got - want).abs())
    bad = ~(off <= bound)
    assert not bad.any(), (
        f"{what}: {int(bad.sum())} of {bad.numel()} values out of bounds, first at "
        f"{tuple(int(x) for x in bad.nonzero()[0])}: {got[bad][0]:.6g}, not {want[bad][0]:.6g} "
        f"+- {bound.expand_as(want)[bad][0]:.2g}")
