"""Cases of the operators that serve many and long texts from the 4-bit cache: new
tokens rotated on their way into it, attention over the pages that a bound on each
page's scores selects, and attention of a batch that shares its first tokens.

``run`` is one pass as a user's program makes it. With ``own`` false the operators
are computed in their plain form (elementary torch operations in 32 bits, in 64
where angles, roundings to 4 bits, interval positions and the order of pages need
them); with ``own`` true through the entry points of ``paper_2609_33591_amd``.
``exact`` gives the same outputs from the definitions in 64 bits.

Sizes are those of this repository's workloads (12 or 24 heads of 64, 16 heads of
128; T = 2048, 8192), fewer key heads than query heads, and single tokens against
caches of 1 000 to 200 000.
"""
import math

import torch

own = False

_APP = dict(op="append", B=1, H=12, Hkv=12, T=1, L=1000, d=64, page=64, rot=64, layout="half",
            scaling="none", split=True, bounds=True, dtype="bf16")
_PAG = dict(op="pages", B=1, H=12, Hkv=12, T=1, L=1000, d=64, page=64, count=8, first=1, last=1,
            recon="softmax", calib="fwm", K=4, tau=8.0, dtype="bf16", ragged=False)
_SHA = dict(op="shared", B=4, H=12, Hkv=12, T=1, S=256, L=50, d=64, page=64, recon="softmax",
            calib="fwm", K=4, tau=8.0, dtype="bf16", ragged=False)


def listed():
    return [
        # one decoding step of 32 sequences: the new token's query rotated, its key and value
        # held, and the bounds of the page that it falls into
        dict(_APP, name="append_token", B=32, H=16, Hkv=4, L=4000, d=128, rot=128),
        # prompts of 2048 tokens, as a projection leaves them ([B, T, heads, d])
        dict(_APP, name="append_prompt", B=4, H=16, Hkv=16, T=2048, L=0, d=128, rot=128),
        # part of a head in neighbouring pairs, stretched frequencies, fp32, odd sizes, and
        # texts that end inside a page before and after
        dict(_APP, name="append_part_f32", B=3, H=5, Hkv=1, T=777, L=5003, page=16, rot=40,
             layout="interleaved", scaling="parts", dtype="f32"),
        # one token of one sequence of a thousand keys: latency
        dict(_PAG, name="pages_token", page=16),
        # serving: 32 sequences of up to 32 000 keys, an eighth of them read, with the interval
        # weights that the model was trained with
        dict(_PAG, name="pages_serve_32k", B=32, H=16, Hkv=4, L=32000, d=128, count=64, recon="lerp",
             K=16, ragged=True),
        # one very long text
        dict(_PAG, name="pages_long_200k", H=16, Hkv=4, L=200000, d=128, count=128, first=2, last=8),
        # four draft tokens in fp32, odd lengths
        dict(_PAG, name="pages_draft_f32", B=5, H=10, Hkv=5, T=4, L=9999, page=32, count=37, last=3,
             recon="lerp", calib="minmax", K=16, dtype="f32", ragged=True),
        # a few sequences behind a short instruction: latency
        dict(_SHA, name="shared_token"),
        # serving: 64 sequences of unequal length behind 8192 tokens of instructions and
        # examples, interval weights
        dict(_SHA, name="shared_serve_8k", B=64, H=16, Hkv=4, S=8192, L=1000, d=128, recon="lerp", K=16,
             ragged=True),
        # many samples of one long prompt
        dict(_SHA, name="shared_wide_16k", B=256, H=16, Hkv=4, S=16384, L=128, d=128),
        # draft tokens in fp32, small pages, odd sizes
        dict(_SHA, name="shared_draft_f32", B=7, H=6, Hkv=2, T=3, S=2048, L=333, page=16, recon="lerp",
             calib="resolved", K=7, dtype="f32", ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng, most):
    hkv = rng.choice([h for h in (1, 2, 3, 4, 5, 8, 12, 16) if h <= most])
    return hkv * rng.choice([g for g in (1, 2, 3, 4, 7, 8) if hkv * g <= most]), hkv


def draw(rng):
    """One more case: sizes spread over the logarithm of their range, and no more work than the
    largest listed case of its kind has."""
    case = _drawn(rng)
    most = {"append": (2e8, 1e12), "pages": (8e7, 1e12), "shared": (2e7, 3e10)}[case["op"]]
    while case["B"] > 1 and (work(case)["bytes"] > most[0] or work(case)["flops"] > most[1]):
        case["B"] //= 2
    return case


def _drawn(rng):
    op = rng.choice(("append", "pages", "shared"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    H, Hkv = _heads(rng, 24)
    d = rng.choice((32, 64, 128))
    page = rng.choice((16, 32, 64, 128, 256))
    if op == "append":
        T = rng.choice((1, 1, 2, 5, _log(rng, 1, 4096)))
        return dict(_APP, B=_log(rng, 1, 48), H=H, Hkv=Hkv, T=T, L=rng.choice((0, 1, _log(rng, 1, 8000))), d=d, page=page,
                    rot=2 * rng.randint(1, d // 2) if rng.random() < 0.4 else d,
                    layout=rng.choice(("half", "interleaved")),
                    scaling=rng.choice(("none", "linear", "base", "parts")), split=rng.random() < 0.6,
                    bounds=rng.random() < 0.7, dtype=dtype)
    # (fp32 results are compared to their last digits: weight functions without a jump)
    recon, calib = rng.choice((("softmax", "fwm"), ("lerp", "minmax"), ("lerp", "resolved"),
                               ("lerp", "fwm") if dtype == "bf16" else ("softmax", "fwm")))
    grid = dict(recon=recon, calib=calib, K=rng.choice((2, 4, 7, 16)), tau=rng.choice((6.0, 8.0)))
    T = rng.choice((1, 1, 1, 2, 5))
    if op == "pages":
        L = _log(rng, 1, 64000)
        first, last = rng.choice((0, 1, 4)), rng.choice((1, 2, 5))
        return dict(_PAG, B=_log(rng, 1, 48), H=H, Hkv=Hkv, T=T, L=L, d=d, page=page,
                    count=first + last + _log(rng, 1, max(2, min(256, 8192 // page))), first=first, last=last,
                    dtype=dtype, ragged=rng.random() < 0.5, **grid)
    S = max(page, 32) * _log(rng, 1, max(2, 16384 // max(page, 32)))
    L = _log(rng, T, 2000)
    B = max(1, min(_log(rng, 1, 256), 134217728 // (H * T * (S + L))))
    return dict(_SHA, B=B, H=H, Hkv=Hkv, T=T, S=S, L=L, d=d, page=page, dtype=dtype,
                ragged=rng.random() < 0.5, **grid)


# ---- inputs -------------------------------------------------------------------
def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _lengths(case):
    """Keys of each sequence after the call; before it, of those that tokens are appended to.
    Ragged: fewer from one sequence to the next."""
    B, n = case["B"], case["L"]
    if case["op"] == "append":  # some end elsewhere in a page
        return [n - (7 * b) % (n // 2 + 1) for b in range(B)]
    if not case["ragged"]:
        lens = [n] * B
    else:
        lens = [max(1, n - (i * n) // B) for i in range(B)]
    return [case["S"] + m for m in lens] if case["op"] == "shared" else lens


def _frequencies(case):
    """Radians per position of each pair, and the rotated values' factor."""
    n, base = case["rot"] // 2, 10000.0
    factor, before = 8.0, 1024.0
    if case["scaling"] == "base":  # a larger base: the slowest pair is stretched by the factor
        base *= factor ** (n / max(1, n - 1))
    f = base ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n)
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "parts":  # pairs that turn often keep their frequency, slow ones are stretched
        keep = ((before * f / (2 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        return f / factor * (1 - keep) + f * keep, 0.1 * math.log(factor) + 1.0
    return f, 1.0


_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_BORDERS = ((0.25, 1), (0.75, 0), (1.25, 1), (1.75, 0), (2.5, 1), (3.5, 0), (5.0, 1))


def _quantised(x):
    """Codes (bit 3 the sign, bits 0-2 the level) and scale bytes of rows of values, in
    groups of 32: the smallest power of two with no value over 6."""
    g = x.unflatten(-1, (-1, 32))
    top, e = torch.frexp(g.abs().amax(-1))
    e = torch.where(top == 0, -126, torch.where(top <= 0.75, e - 3, e - 2)).clamp(-126, 125)
    a = torch.ldexp(g.abs(), -e[..., None])
    c = sum((a > t if up else a >= t).to(torch.uint8) for t, up in _BORDERS)
    return (c | (torch.signbit(g).to(torch.uint8) << 3)).reshape(x.shape), (e + 127).to(torch.uint8)


def _values(codes, scales):
    """What codes and scale bytes stand for, fp32."""
    level = torch.tensor(_LEVELS + tuple(-v for v in _LEVELS), device=codes.device)
    s = torch.ldexp(torch.ones((), device=codes.device), scales.to(torch.int32) - 127)
    return (level[codes.long()].unflatten(-1, (-1, 32)) * s[..., None]).reshape(codes.shape)


def _key_parts(data, d):
    """Key codes [..., page, d / 2] and scales [..., page, d / 32] of blocks [..., bytes]."""
    page = data.shape[-1] // (d // 2 + d // 32)
    return (data[..., :page * d // 2].unflatten(-1, (page, -1)),
            data[..., page * d // 2:].unflatten(-1, (page, -1)))


def _value_parts(data, d):
    """Value codes [..., page / 4, 16, 4, d / 32] (four tokens' shares of a column block side by
    side) and scales [..., page / 4, d / 32, 4]."""
    page = data.shape[-1] // (d // 2 + d // 32)
    return (data[..., :page * d // 2].unflatten(-1, (page // 4, 16, 4, -1)),
            data[..., page * d // 2:].unflatten(-1, (page // 4, -1, 4)))


def _pairs(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _nibbles(b):
    return torch.stack((b & 15, b >> 4), -1).flatten(-2)


def _keys(data, d):
    """Keys [..., page, d] of blocks [..., bytes], fp32."""
    kb, ks = _key_parts(data, d)
    return _values(_nibbles(kb), ks)


def _vals(data, d):
    vb, vs = _value_parts(data, d)
    return _values(_nibbles(vb.transpose(-2, -3).flatten(-2)).flatten(-3, -2),
                   vs.transpose(-1, -2).flatten(-3, -2))


def _cache(case, used, g):
    """A cache of random tokens: keys with a few larger channels and with what the tokens of a
    page have in common, as trained models have. For pages without tokens, anything."""
    d, page, Hkv = case["d"], case["page"], case["Hkv"]
    data = torch.empty((used, 2, Hkv, page * (d // 2 + d // 32)), dtype=torch.uint8, device="cuda")
    for h in range(Hkv):
        k, v = (torch.randn((used, page, d), generator=g, device="cuda") for _ in range(2))
        k += 0.7 * torch.randn((used, 1, d), generator=g, device="cuda")
        k[..., ::16] *= 2.5
        (kc, ks), (vc, vs) = _quantised(k), _quantised(v)
        for part, x in zip(_key_parts(data[:, 0, h], d) + _value_parts(data[:, 1, h], d), (
                _pairs(kc), ks, _pairs(vc).unflatten(-2, (page // 4, 4)).unflatten(-1, (16, -1)).transpose(2, 3),
                vs.unflatten(-2, (page // 4, 4)).transpose(-1, -2))):
            part.copy_(x)
    return data


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 31)
    t, B, T, d, page, Hkv = _type(case), case["B"], case["T"], case["d"], case["page"], case["Hkv"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(t)

    # each sequence's pages anywhere in the cache, unused entries of the table -1; the shared
    # tokens' pages first, the same for all
    lens = _lengths(case)
    s = dict(case=case, lengths=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    common = case["S"] // page if case["op"] == "shared" else 0
    ends = [n + T for n in lens] if case["op"] == "append" else lens
    need = [(n + page - 1) // page - common for n in ends]
    used = common + sum(need) + 3
    place = torch.randperm(used, generator=g, device="cuda").to(torch.int32)
    need = torch.tensor(need, device="cuda")
    i = torch.arange(int(need.max()), device="cuda")
    at = (common + torch.cumsum(need, 0) - need)[:, None] + i
    tail = torch.where(i < need[:, None], place[at.clamp(max=used - 1)], -1)
    s["table"] = torch.cat((place[:common].expand(B, common), tail), 1).contiguous()
    s["cache"] = _cache(case, used, g)
    if case["op"] == "append":
        for n, heads in (("q", case["H"]), ("k", Hkv), ("v", Hkv)):
            s[n] = normal(B, T, heads, d).transpose(1, 2) if case["split"] else normal(B, heads, T, d)
        s["freq"], s["factor"] = _frequencies(case)
        s["bounds"] = torch.zeros((used, Hkv, 2, d), dtype=torch.bfloat16, device="cuda")
        return s
    s["q"] = normal(B, case["H"], T, d)
    if case["op"] == "pages":  # (a page's bounds are over its tokens; of the last page over all of
        # them that it has room for, which a rewound text leaves too)
        s["bounds"] = torch.empty((used, Hkv, 2, d), dtype=torch.bfloat16, device="cuda")
        for h in range(Hkv):
            k = _keys(s["cache"][:, 0, h], d)
            s["bounds"][:, h, 0], s["bounds"][:, h, 1] = k.amin(1), k.amax(1)
    return s


# ---- the operators in their plain form ------------------------------------------
def _turned(x, cos, sin, case):
    n, f = case["rot"] // 2, x.double()
    r = f[..., :2 * n]
    if case["layout"] == "half":
        a, b = r[..., :n], r[..., n:]
        r = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((r, f[..., 2 * n:]), -1)


def _plain_append(s):
    case, page, d, T = s["case"], s["case"]["page"], s["case"]["d"], s["case"]["T"]
    pos = s["lengths"].long()[:, None] + torch.arange(T, device="cuda")
    angle = pos.double()[:, None, :, None] * s["freq"]
    cos, sin = torch.cos(angle) * s["factor"], torch.sin(angle) * s["factor"]
    out = {"q": _turned(s["q"], cos, sin, case).to(s["q"].dtype)}
    pages, at = torch.gather(s["table"].long(), 1, pos // page), pos % page  # [B, T]
    (kb, ks), (vb, vs) = _key_parts(s["cache"][:, 0], d), _value_parts(s["cache"][:, 1], d)
    kc, kn = _quantised(_turned(s["k"], cos, sin, case).transpose(1, 2))
    vc, vn = _quantised(s["v"].float().transpose(1, 2))
    kb[pages, :, at], ks[pages, :, at] = _pairs(kc), kn
    vb[pages, :, at // 4, :, at % 4] = _pairs(vc).unflatten(-1, (16, -1))
    vs[pages, :, at // 4, :, at % 4] = vn
    k = _values(_nibbles(kb[pages, :, at]), ks[pages, :, at])
    v = _values(_nibbles(vb[pages, :, at // 4, :, at % 4]).flatten(-2), vs[pages, :, at // 4, :, at % 4])
    out["k"], out["v"] = k.transpose(1, 2).to(s["k"].dtype), v.transpose(1, 2).to(s["v"].dtype)
    if case["bounds"]:
        end = s["lengths"].long() + T
        i = s["lengths"].long()[:, None] // page + torch.arange((T + page - 2) // page + 1, device="cuda")
        i = torch.minimum(i, ((end - 1) // page)[:, None])
        held = torch.gather(s["table"].long(), 1, i)
        k = _keys(s["cache"][held, 0], d)  # [B, n, Hkv, page, d]
        here = (i[..., None] * page + torch.arange(page, device="cuda") < end[:, None, None])[:, :, None, :, None]
        s["bounds"][held, :, 0] = k.masked_fill(~here, math.inf).amin(-2).bfloat16()
        s["bounds"][held, :, 1] = k.masked_fill(~here, -math.inf).amax(-2).bfloat16()
        out["bounds"] = s["bounds"]
    return out


def _weights(z, see, case):
    """Weights of scores z for the keys that each row sees, and the sum over a row."""
    top = z.masked_fill(~see, -math.inf).amax(-1, keepdim=True)
    if case["recon"] == "softmax":
        w = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    else:
        K, tau = case["K"], case["tau"]
        low = z.masked_fill(~see, math.inf).amin(-1, keepdim=True)
        span = top.double() - low.double() if case["calib"] == "minmax" else \
            torch.full_like(top, tau).double()
        u = K * ((z.double() - top.double()) + span) / span.clamp(min=1e-30)
        r = u.floor().clamp(max=K - 1)
        t = (u - r).clamp(0, 1)
        e = lambda b: torch.exp(b / K * span - span).float()  # noqa: E731
        w = (1 - t).float() * e(r) + t.float() * e(r + 1)
        if case["calib"] == "fwm":
            w = torch.where(u < 0, 0.0, w)
        if case["calib"] == "minmax":
            w = torch.where(span <= 1e-12, 1.0, w)
    w = w.masked_fill(~see, 0.0)
    total = w.sum(-1, keepdim=True)
    return w, torch.where(total == 0, 1.0, total)


def _position(s):
    """The new tokens' positions [B, T]."""
    T = s["case"]["T"]
    return s["lengths"].long()[:, None] - T + torch.arange(T, device="cuda")


def _plain_pages(s):
    case, d, page, Hkv = s["case"], s["case"]["d"], s["case"]["page"], s["case"]["Hkv"]
    B, H, T, _ = s["q"].shape
    G, W = H // Hkv, s["table"].shape[1]
    q = s["q"].reshape(B, Hkv, G * T, d)
    bounds = s["bounds"][s["table"].long().clamp(min=0)].double().transpose(1, 2)  # [B, Hkv, W, 2, d]
    score = torch.matmul(q.double().clamp(min=0), bounds[:, :, :, 1].transpose(-1, -2)) + \
        torch.matmul(q.double().clamp(max=0), bounds[:, :, :, 0].transpose(-1, -2))
    score = score.reshape(B, Hkv, G, T, W).amax(2)
    i, w = _position(s)[:, None, :, None], torch.arange(W, device="cuda")
    here = (w * page <= i) & (s["table"] >= 0)[:, None, None]
    score = torch.where((w < case["first"]) | (w > i // page - case["last"]), math.inf, score)
    score = score.masked_fill(~here, -math.inf)
    n = min(case["count"], W)
    best, order = (x[..., :n] for x in torch.sort(score, descending=True, stable=True))
    order = torch.where(best == -math.inf, W, order).sort(-1).values
    pages = torch.nn.functional.pad(torch.where(order == W, -1, order), (0, case["count"] - n), value=-1)
    held = torch.gather(s["table"].long()[:, None, None].expand(B, Hkv, T, W), 3, order.clamp(max=W - 1))
    heads = torch.arange(Hkv, device="cuda")[:, None, None]
    k, v = _keys(s["cache"][held, 0, heads], d).flatten(3, 4), _vals(s["cache"][held, 1, heads], d).flatten(3, 4)
    at = (order[..., None] * page + torch.arange(page, device="cuda")).flatten(-2)  # [B, Hkv, T, n page]
    see = ((at <= i) & (order < W).repeat_interleave(page, -1))[..., None, :]
    q = s["q"].float().reshape(B, Hkv, G, T, d).transpose(2, 3)
    w, total = _weights(torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(d)), see, case)
    o = torch.matmul(w, v) / total
    return {"pages": pages.to(torch.int32), "o": o.transpose(2, 3).reshape(B, H, T, d).to(s["q"].dtype)}


def _plain_shared(s):
    case, d, page, S, Hkv = s["case"], s["case"]["d"], s["case"]["page"], s["case"]["S"], s["case"]["Hkv"]
    B, H, T, _ = s["q"].shape
    G, n = H // Hkv, S // page
    q = s["q"].float().reshape(B, Hkv, G * T, d)
    i = _position(s).repeat(1, G)[:, None, :, None]  # [B, 1, G T, 1]
    data = s["cache"][s["table"][0, :n].long()].transpose(0, 2)  # [Hkv, 2, n, bytes]
    k0, v0 = _keys(data[:, 0], d).flatten(1, 2), _vals(data[:, 1], d).flatten(1, 2)  # [Hkv, S, d]
    data = s["cache"][s["table"][:, n:].long().clamp(min=0)].transpose(1, 3)  # [B, Hkv, 2, n', bytes]
    k1, v1 = _keys(data[:, :, 0], d).flatten(2, 3), _vals(data[:, :, 1], d).flatten(2, 3)
    rows = q.transpose(0, 1).reshape(Hkv, B * G * T, d)
    z0 = torch.matmul(rows, k0.transpose(-1, -2)).reshape(Hkv, B, G * T, S).transpose(0, 1)
    z = torch.cat((z0, torch.matmul(q, k1.transpose(-1, -2))), -1) * (1.0 / math.sqrt(d))
    j = torch.arange(z.shape[-1], device="cuda")
    w, total = _weights(z, (j <= i) & (i >= 0), case)
    o = torch.matmul(w[..., :S].transpose(0, 1).reshape(Hkv, B * G * T, S), v0)
    o = o.reshape(Hkv, B, G * T, d).transpose(0, 1) + torch.matmul(w[..., S:], v1)
    return {"o": (o / total).reshape(B, H, T, d).to(s["q"].dtype)}


# ---- the calls of the framework ----------------------------------------------------
def _own(s):
    import paper_2609_33591_amd as kia

    case = s["case"]
    cache = kia.Cache4(s["cache"], case["d"])
    if case["op"] == "append":
        plan = kia.RotaryPlan(s["freq"], layout=case["layout"], factor=s["factor"])
        bounds = s["bounds"] if case["bounds"] else None
        out = {"q": kia.cache4_append(s["q"], s["k"], s["v"], cache, s["table"], s["lengths"], plan, bounds=bounds)}
        out["k"], out["v"] = kia.cache4_read(cache, s["table"], s["lengths"], case["T"], s["k"].dtype)
        if case["bounds"]:
            out["bounds"] = bounds
        return out
    grid = dict(K=case["K"], calib=case["calib"], tau=case["tau"], recon=case["recon"])
    if case["op"] == "pages":
        pages = kia.cache4_select(s["q"], cache, s["bounds"], s["table"], s["lengths"], case["count"],
                                  first=case["first"], last=case["last"])
        return {"pages": pages,
                "o": kia.cache4_attention(s["q"], cache, s["table"], s["lengths"], pages=pages, **grid)}
    return {"o": kia.cache4_attention(s["q"], cache, s["table"], s["lengths"], shared=case["S"], **grid)}


def run(s):
    if own:
        return _own(s)
    return {"append": _plain_append, "pages": _plain_pages, "shared": _plain_shared}[s["case"]["op"]](s)


def work(case):
    i, d, B, T, H, Hkv, page = (4 if case["dtype"] == "f32" else 2), case["d"], case["B"], case["T"], \
        case["H"], case["Hkv"], case["page"]
    lens = _lengths(case)
    token = 2 * Hkv * d * 17 // 32  # bytes that a token's key and value take
    if case["op"] == "append":  # read, written, held, held read back, written
        n = B * T * d
        old = sum(m % page for m in lens) if case["bounds"] else 0  # the bounds' earlier keys
        pages = sum((m + T + page - 1) // page - m // page for m in lens) if case["bounds"] else 0
        return {"bytes": i * n * (2 * H + 4 * Hkv) + 2 * B * T * token + old * token // 2 + 4 * pages * Hkv * d,
                "flops": 3 * n * (H + Hkv) * case["rot"] // d + 2 * n * Hkv}
    io = 2 * i * B * H * T * d
    if case["op"] == "pages":
        pages = keys = 0
        for n in lens:
            for t in range(max(0, n - T), n):
                have = t // page + 1
                keys += min(case["count"], have) * page if have > case["count"] else t + 1
            pages += (n + page - 1) // page
        return {"bytes": 4 * pages * Hkv * d + keys * token + io,
                "flops": 2 * T * H * d * pages + 4 * H * d * keys}
    keys = sum(n - case["S"] for n in lens)
    return {"bytes": (case["S"] + keys) * token + io, "flops": 4 * H * T * d * (B * case["S"] + keys)}


# ---- 64 bits ------------------------------------------------------------------------
def _exact_turned(x, s, pos):
    """As a product of complex numbers."""
    case, t = s["case"], x.double().clone()
    n = case["rot"] // 2
    turn = torch.polar(torch.full_like(s["freq"], s["factor"]).expand(*pos.shape, n),
                       pos.double()[..., None] * s["freq"])[:, None]
    if case["layout"] == "half":
        z = torch.complex(t[..., :n], t[..., n:2 * n]) * turn
        t[..., :n], t[..., n:2 * n] = z.real, z.imag
    else:
        z = torch.view_as_complex(t[..., :2 * n].reshape(*t.shape[:-1], n, 2).contiguous()) * turn
        t[..., 0:2 * n:2], t[..., 1:2 * n:2] = z.real, z.imag
    return t


def _exact_held(x):
    """The nearest of the 15 values at the group's scale, an even code between two."""
    g = x.double().reshape(*x.shape[:-1], -1, 32)
    top = g.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -130) / 6)) - 1
    for _ in range(3):
        e = torch.where(top > 6 * torch.exp2(e), e + 1, e)
    s = torch.exp2(e.clamp(-126, 125))
    level = torch.tensor(_LEVELS, dtype=torch.float64, device=x.device)
    a, near = g.abs() / s, torch.zeros_like(g)
    for n in range(7):  # past the midpoint to the next level, or on it where that is the even one
        mid = (level[n] + level[n + 1]) / 2
        near = torch.where((a >= mid) if n % 2 else (a > mid), level[n + 1], near)
    return torch.copysign(near * s, g).reshape(x.shape)


def _exact_block(block, d, value):
    """Keys or values [page, d] of one head's block, nibble by nibble."""
    page = block.numel() // (d // 2 + d // 32)
    t, c = torch.arange(page, device="cuda")[:, None], torch.arange(d, device="cuda")
    if value:
        r, low = c // (d // 16), c % (d // 16)
        byte = t // 4 * (2 * d) + r * (d // 8) + t % 4 * (d // 32) + low // 2
        scale = page * d // 2 + t // 4 * (d // 8) + c // 32 * 4 + t % 4
    else:
        byte, scale = t * (d // 2) + c // 2, page * d // 2 + t * (d // 32) + c // 32
    code = (block[byte].long() >> (4 * (c % 2))) & 15
    x = torch.tensor(_LEVELS, dtype=torch.float64, device="cuda")[code & 7]
    return torch.where(code >= 8, -x, x) * torch.exp2(block[scale].double() - 127)


def _exact_append(case, s):
    B, T, d, page, Hkv = case["B"], case["T"], case["d"], case["page"], case["Hkv"]
    lens = _lengths(case)
    pos = torch.tensor(lens, device="cuda")[:, None] + torch.arange(T, device="cuda")
    out = {"q": _exact_turned(s["q"], s, pos), "k": _exact_held(_exact_turned(s["k"], s, pos)),
           "v": _exact_held(s["v"])}
    if case["bounds"]:
        out["bounds"] = torch.zeros(s["bounds"].shape, dtype=torch.float64, device="cuda")
        table = s["table"].tolist()
        for b, n in enumerate(lens):
            for w in range(n // page, (n + T - 1) // page + 1):
                lo, hi = max(n, w * page), min(n + T, w * page + page)
                new = out["k"][b, :, lo - n:hi - n]
                old = [_exact_block(s["cache"][table[b][w], 0, h], d, False)[:lo - w * page] for h in range(Hkv)]
                every = torch.cat((torch.stack(old), new), 1)
                out["bounds"][table[b][w], :, 0], out["bounds"][table[b][w], :, 1] = every.amin(1), every.amax(1)
    return out


def _exact_row(q, k, v, case):
    """One token's queries [G, d] of a key head over the keys and values that they see."""
    z = (q @ k.T) / math.sqrt(case["d"])
    z = z - z.amax(-1, keepdim=True)
    if case["recon"] == "softmax":
        w = torch.exp(z)
    else:
        K = case["K"]
        h = -z.amin(-1, keepdim=True) / K if case["calib"] == "minmax" else \
            torch.full_like(z[..., :1], case["tau"] / K)
        same = h * K <= 1e-12
        h = torch.where(same, 1.0, h)
        low = torch.floor((z / h).clamp(max=-1e-300)).clamp(max=-1.0)  # interval [low, low + 1] h
        part = z / h - low
        w = torch.exp(low * h) * (1 - part) + torch.exp((low + 1) * h) * part
        w = torch.where(same, 1.0, w)
        if case["calib"] == "fwm":
            w = torch.where(z < -case["tau"], 0.0, w)
    return (w / w.sum(-1, keepdim=True)) @ v


def _exact_served(case, s):
    """Token by token and key head by key head: the row of its visible keys alone."""
    d, page, T, Hkv = case["d"], case["page"], case["T"], case["Hkv"]
    q, G = s["q"].double(), case["H"] // case["Hkv"]
    out = {"o": torch.zeros_like(q)}
    if case["op"] == "pages":
        out["pages"] = torch.full((case["B"], Hkv, T, case["count"]), -1, dtype=torch.int32, device="cuda")
    table, shared = s["table"].tolist(), {}
    for b, n in enumerate(_lengths(case)):
        for h in range(Hkv):
            def block(w):
                mine = shared if w * page < case.get("S", 0) else {}
                if (w, h) not in mine:
                    mine[w, h] = [_exact_block(s["cache"][table[b][w], i, h], d, i == 1) for i in (0, 1)]
                return mine[w, h]

            whole = None
            for t in range(max(0, T - n), T):
                i = n - T + t
                x = q[b, h * G:h * G + G, t]
                ws = list(range(i // page + 1))
                if case["op"] == "pages" and len(ws) > case["count"]:
                    lo, hi = s["bounds"][table[b][:len(ws)], h].double().unbind(1)
                    score = torch.maximum(x[:, None] * lo, x[:, None] * hi).sum(-1).amax(0).tolist()
                    must = [w for w in ws if w < case["first"] or w > i // page - case["last"]]
                    rest = sorted((w for w in ws if w not in set(must)), key=lambda w: (-score[w], w))
                    ws = sorted(must + rest[:case["count"] - len(must)])
                if case["op"] == "pages":
                    out["pages"][b, h, t, :len(ws)] = torch.tensor(ws, dtype=torch.int32)
                    data = [block(w) for w in ws]
                else:  # (the later tokens see the earlier ones' keys and more)
                    whole = whole or [block(w) for w in range((n - 1) // page + 1)]
                    data = whole[:len(ws)]
                k, v = (torch.cat([p[m] for p in data]) for m in (0, 1))
                see = torch.cat([w * page + torch.arange(page, device="cuda") for w in ws]) <= i
                out["o"][b, h * G:h * G + G, t] = _exact_row(x, k[see], v[see], case)
    return out


def exact(case, seed):
    # (page by page on the host's pace: not where there are too many)
    if case["op"] == "pages":
        pages = case["B"] * case["Hkv"] * case["T"] * min(case["count"], case["L"] // case["page"] + 1)
    elif case["op"] == "shared":
        pages = case["Hkv"] * (case["S"] // case["page"] + case["B"] * (case["L"] // case["page"] + 1))
    else:
        pages = case["B"] * case["Hkv"] * (case["T"] // case["page"] + 2)
    if pages > 20000:
        return None
    s = prepare(case, seed)
    return _exact_append(case, s) if case["op"] == "append" else _exact_served(case, s)
