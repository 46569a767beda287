"""Cases of the operators around K-interval attention: rotary positions, softmax
attention with a sliding window and visible first tokens, a paged key/value
cache held in 4 bits, and attention of new tokens over that cache.

``run`` is one pass as a user's program makes it. With ``own`` false the
operators are computed in their plain form (elementary torch operations in 32
bits, in 64 where angles or interval positions need them); with ``own`` true
through the entry points of ``paper_2609_33591_amd``. ``exact`` gives the same
outputs from the definitions in 64 bits.

Sizes are those of this repository's workloads (12 or 24 heads of 64, 16 heads
of 128; T = 1024, 2048, 8192), fewer key heads than query heads, and single
tokens against caches of 1 000 to 32 000.
"""
import math

import torch

own = False

_ROT = dict(op="rotary", B=1, H=12, Hkv=12, T=1024, d=64, rot=64, layout="half", scaling="none",
            dtype="bf16", far=0, split=False, grad=False)
_WIN = dict(op="window", B=1, H=12, Hkv=12, T=1024, d=64, window=256, sinks=4, dtype="bf16",
            ragged=False, grad=True)
_WR = dict(op="write", B=1, Hkv=12, T=1, L=1024, d=64, page=64, dtype="bf16")
_ATT = dict(op="cached", B=1, H=12, Hkv=12, T=1, L=1024, d=64, page=64, window=0, sinks=0,
            recon="softmax", calib="fwm", K=4, tau=8.0, dtype="bf16", ragged=False)


def listed():
    return [
        # one decoding step of 16 sequences far into their text: launch latency
        dict(_ROT, name="rotary_token", B=16, H=24, Hkv=24, T=1, far=100000),
        # positions in a training step at 1B scale: q and k as a projection leaves them
        # ([B, T, H, d]), rotated, and their gradients rotated back
        dict(_ROT, name="rotary_train_1b", B=4, H=16, Hkv=16, T=2048, d=128, rot=128, split=True,
             grad=True),
        # part of a head, neighbouring pairs, frequencies stretched for a longer
        # context, fp32, odd sizes
        dict(_ROT, name="rotary_part_f32", B=3, H=5, Hkv=1, T=777, rot=40, layout="interleaved",
             scaling="parts", dtype="f32", far=5000, grad=True),
        # unit test size, fp32, window and sinks inside one tile
        dict(_WIN, name="window_tiny_f32", H=2, Hkv=1, T=65, d=32, window=20, sinks=2,
             dtype="f32"),
        # a training step of a local layer at 1B scale, four query heads to a key head
        dict(_WIN, name="window_train_1b", B=4, H=16, Hkv=4, T=2048, d=128, window=512),
        # a padded batch in fp32 with a sequence of length 0
        dict(_WIN, name="window_ragged_f32", B=4, H=6, Hkv=2, T=777, window=200, sinks=3,
             dtype="f32", ragged=True),
        # the prompt of a long text (T = 8192, 16 heads of 128), forward only
        dict(_WIN, name="window_prompt_8k", H=16, Hkv=4, T=8192, d=128, window=1024, sinks=16,
             grad=False),
        # the key and value of one new token of 32 sequences into the cache, and
        # what the cache then holds of them
        dict(_WR, name="cache_token", B=32, Hkv=8, L=4000, d=128),
        # a prompt of 2048 tokens into the cache, and read back
        dict(_WR, name="cache_prompt", B=4, Hkv=16, T=2048, L=0, d=128),
        # one token of one sequence, 12 heads of 64, a thousand keys: latency
        dict(_ATT, name="cached_token", L=1000),
        # serving: 32 sequences of up to 32 000 keys, four query heads to a key
        # head, the interval weights that the model was trained with
        dict(_ATT, name="cached_serve_32k", B=32, H=16, Hkv=4, L=32000, d=128, recon="lerp", K=16,
             ragged=True),
        # four draft tokens in fp32 over a window and first tokens of a long cache,
        # odd lengths and small pages
        dict(_ATT, name="cached_window_f32", B=8, H=10, Hkv=5, T=4, L=9999, d=64, page=16,
             window=4000, sinks=5, dtype="f32", ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng, most):
    hkv = rng.choice([h for h in (1, 2, 3, 4, 5, 8, 12, 16) if h <= most])
    return hkv * rng.choice([g for g in (1, 2, 3, 4, 7, 8) if hkv * g <= most]), hkv


def draw(rng):
    """One more case: sizes spread over the logarithm of their range."""
    op = rng.choice(("rotary", "window", "window", "write", "cached", "cached"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    B = _log(rng, 1, 16)
    H, Hkv = _heads(rng, 24)
    if op == "rotary":
        d = rng.choice((16, 32, 64, 128))
        T = min(_log(rng, 1, 4096), max(1, 16777216 // (B * H * d)))
        return dict(_ROT, B=B, H=H, Hkv=Hkv, T=T, d=d, rot=2 * rng.randint(1, d // 2)
                    if rng.random() < 0.4 else d, layout=rng.choice(("half", "interleaved")),
                    scaling=rng.choice(("none", "linear", "base", "parts")), dtype=dtype,
                    far=rng.choice((0, 0, 3000, 120000)), split=rng.random() < 0.5,
                    grad=rng.random() < 0.5)
    if op == "window":
        d = rng.choice((16, 32, 64, 128))
        T = _log(rng, 1, 6000 if dtype == "bf16" else 2000)
        B = max(1, min(B, 268435456 // (H * T * T)))
        # (a row that sees itself alone has gradients of 0, which say nothing)
        return dict(_WIN, B=B, H=H, Hkv=Hkv, T=T, d=d, window=_log(rng, 2, 2 * T + 2),
                    sinks=rng.choice((0, 1, 4, 16, 100)), dtype=dtype, ragged=rng.random() < 0.4,
                    grad=T >= 8 and rng.random() < 0.7)
    d = rng.choice((32, 64, 128))
    page = rng.choice((16, 32, 64, 128))
    if op == "write":
        T = min(_log(rng, 1, 4096), max(1, 16777216 // (B * Hkv * d)))
        return dict(_WR, B=B, Hkv=Hkv, T=T, L=rng.choice((0, 1, 77, 1000)), d=d, page=page,
                    dtype=dtype)
    T = rng.choice((1, 1, 1, 2, 5))
    L = _log(rng, 1, 32000)
    B = max(1, min(B, 4194304 // (H * T * L) * 4))
    # (fp32 results are compared to their last digits: weight functions without a jump)
    recon, calib = rng.choice((("softmax", "fwm"), ("lerp", "minmax"), ("lerp", "resolved"),
                               ("lerp", "fwm") if dtype == "bf16" else ("softmax", "fwm")))
    window = rng.choice((0, 0, _log(rng, 1, L)))
    return dict(_ATT, B=B, H=H, Hkv=Hkv, T=T, L=L, d=d, page=page, window=window,
                sinks=rng.choice((0, 3, 64)) if window else 0, recon=recon, calib=calib,
                K=rng.choice((2, 4, 7, 16)), tau=rng.choice((6.0, 8.0)), dtype=dtype,
                ragged=rng.random() < 0.5)


# ---- inputs -------------------------------------------------------------------
def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _lengths(case):
    """Keys of each sequence: all of them or, in a ragged batch, fewer from one to
    the next; a padded training batch ends with an empty sequence."""
    B, n = case["B"], case["T"] if case["op"] == "window" else case["L"] + case["T"] - 1
    if not case["ragged"]:
        return [n] * B
    lens = [n - (i * n) // B for i in range(B)]
    if case["op"] == "window" and B > 2:
        lens[-1] = 0
    return lens


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
        turns = before * f / (2 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        return f / factor * (1 - keep) + f * keep, 0.1 * math.log(factor) + 1.0
    return f, 1.0


_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantised(x):
    """Codes (bit 3 the sign, bits 0-2 the level) and scale bytes of rows of fp32
    values, in groups of 32: the smallest power of two with no value over 6."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    top, e = torch.frexp(g.abs().amax(-1))
    e = torch.where(top == 0, -126, torch.where(top <= 0.75, e - 3, e - 2)).clamp(-126, 125)
    a = torch.ldexp(g.abs(), -e[..., None])
    c = sum((a > t if up else a >= t).to(torch.uint8)
            for t, up in ((0.25, 1), (0.75, 0), (1.25, 1), (1.75, 0), (2.5, 1), (3.5, 0), (5.0, 1)))
    return (c | (torch.signbit(g).to(torch.uint8) << 3)).reshape(x.shape), (e + 127).to(torch.uint8)


def _values(codes, scales):
    """What codes and scale bytes stand for, fp32."""
    level = torch.tensor(_LEVELS + tuple(-v for v in _LEVELS), device=codes.device)
    s = torch.ldexp(torch.ones((), device=codes.device), scales.to(torch.int32) - 127)
    g = level[codes.long()].reshape(*codes.shape[:-1], -1, 32)
    return (g * s[..., None]).reshape(codes.shape)


def _packed(k, v, page):
    """Rows [n, page, d] of one key head's pages, as the cache lays them out: keys
    by token, values with four tokens' shares of a column block side by side."""
    n, _, d = k.shape
    (kc, ks), (vc, vs) = _quantised(k), _quantised(v)
    kb = kc[..., 0::2] | (kc[..., 1::2] << 4)
    vb = (vc[..., 0::2] | (vc[..., 1::2] << 4)).reshape(n, page // 4, 4, 16, d // 32)
    vs = vs.reshape(n, page // 4, 4, d // 32).transpose(2, 3)
    flat = [t.reshape(n, -1) for t in (kb, ks, vb.transpose(2, 3), vs)]
    return torch.cat(flat[:2], 1), torch.cat(flat[2:], 1)


def _views(data, d):
    """The four parts of pages [..., 2, Hkv, bytes]: key codes [..., page, d / 2], key scales
    [..., page, d / 32], value codes [..., page / 4, 16, 4, d / 32] and value scales
    [..., page / 4, d / 32, 4]."""
    page = data.shape[-1] // (d // 2 + d // 32)
    part = lambda x: (x[..., :page * d // 2], x[..., page * d // 2:])  # noqa: E731
    (kb, ks), (vb, vs) = part(data.select(-3, 0)), part(data.select(-3, 1))
    return (kb.unflatten(-1, (page, -1)), ks.unflatten(-1, (page, -1)),
            vb.unflatten(-1, (page // 4, 16, 4, -1)), vs.unflatten(-1, (page // 4, -1, 4)))


def _nibbles(b):
    return torch.stack((b & 15, b >> 4), -1).flatten(-2)


def _unpacked(data, d):
    """Pages [..., 2, Hkv, bytes] as keys and values [..., Hkv, page, d] in fp32."""
    kb, ks, vb, vs = _views(data, d)
    vc = _nibbles(vb.transpose(-2, -3).flatten(-2)).flatten(-3, -2)
    return _values(_nibbles(kb), ks), _values(vc, vs.transpose(-1, -2).flatten(-3, -2))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 29)
    t, B, T, d = _type(case), case["B"], case["T"], case["d"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(t)

    s = dict(case=case)
    if case["op"] == "rotary":
        for n, heads in (("q", case["H"]), ("k", case["Hkv"]), ("dq", case["H"]), ("dk", case["Hkv"])):
            s[n] = normal(B, T, heads, d).transpose(1, 2) if case["split"] else normal(B, heads, T, d)
        first = torch.randint(0, case["far"] + 1, (B, 1), generator=g, device="cuda")
        s["positions"] = (first + torch.arange(T, device="cuda")).to(torch.int32)
        s["freq"], s["factor"] = _frequencies(case)
        return s
    if case["op"] == "window":
        for n, heads in (("q", case["H"]), ("k", case["Hkv"]), ("v", case["Hkv"]), ("dO", case["H"])):
            s[n] = normal(B, heads, T, d)
        s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") \
            if case["ragged"] else None
        return s
    # the cache: each sequence's pages anywhere in it, unused entries of the table -1
    Hkv, page = case["Hkv"], case["page"]
    lens = _lengths(case) if case["op"] == "cached" else [case["L"] + T] * B
    per = (max(lens) + page - 1) // page
    used = sum((n + page - 1) // page for n in lens)
    place = torch.randperm(used + 3, generator=g, device="cuda").to(torch.int32)
    need = torch.tensor([(n + page - 1) // page for n in lens], device="cuda")
    i = torch.arange(per, device="cuda")
    at = (torch.cumsum(need, 0) - need)[:, None] + i
    s["table"] = torch.where(i < need[:, None], place[at.clamp(max=used + 2)], -1).contiguous()
    size = page * (d // 2 + d // 32)
    s["cache"] = torch.zeros((used + 3, 2, Hkv, size), dtype=torch.uint8, device="cuda")
    if case["op"] == "write":
        s["k"], s["v"] = normal(B, Hkv, T, d), normal(B, Hkv, T, d)
        s["starts"] = torch.full((B,), case["L"], dtype=torch.int32, device="cuda")
        return s
    for h in range(Hkv):  # keys with a few larger channels, as trained models have
        k, v = (torch.randn((used + 3, page, d), generator=g, device="cuda") for _ in range(2))
        k[..., ::16] *= 3.0
        s["cache"][:, 0, h], s["cache"][:, 1, h] = _packed(k, v, page)
    s["q"] = normal(B, case["H"], T, d)
    s["lengths"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    return s


# ---- the operators in their plain form ------------------------------------------
def _plain_rotary(x, s, back):
    case = s["case"]
    n = case["rot"] // 2
    angle = s["positions"].double()[:, None, :, None] * s["freq"]
    cos, sin = (torch.cos(angle) * s["factor"]).float(), (torch.sin(angle) * s["factor"]).float()
    sin = -sin if back else sin
    f = x.float()
    r = f[..., :2 * n]
    if case["layout"] == "half":
        a, b = r[..., :n], r[..., n:]
        r = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((r, f[..., 2 * n:]), -1).to(x.dtype)


def _plain_window(s):
    case, q, k, v = s["case"], s["q"].float(), s["k"].float(), s["v"].float()
    B, H, T, d = q.shape
    Hkv, scale = case["Hkv"], 1.0 / math.sqrt(case["d"])
    q = q.reshape(B, Hkv, H // Hkv, T, d)
    i, j = torch.arange(T, device="cuda")[:, None], torch.arange(T, device="cuda")
    see = (j <= i) & ((i - j < case["window"]) | (j < case["sinks"]))
    if s["lengths"] is not None:
        n = s["lengths"].reshape(B, 1, 1, 1, 1)
        see = see & (i < n) & (j < n)
    z = (torch.matmul(q, k[:, :, None].transpose(-1, -2)) * scale).masked_fill(~see, -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    o = torch.matmul(p, v[:, :, None])
    out = {"o": o.reshape(B, H, T, d).to(s["q"].dtype),
           "lse": (top + torch.log(total)).reshape(B, H, T)}
    if case["grad"]:
        g = s["dO"].float().reshape(B, Hkv, H // Hkv, T, d)
        dz = p * (torch.matmul(g, v[:, :, None].transpose(-1, -2)) - (g * o).sum(-1, keepdim=True))
        out["dq"] = (torch.matmul(dz, k[:, :, None]) * scale).reshape(B, H, T, d).to(s["q"].dtype)
        out["dk"] = (torch.matmul(dz.transpose(-1, -2), q).sum(2) * scale).to(s["q"].dtype)
        out["dv"] = torch.matmul(p.transpose(-1, -2), g).sum(2).to(s["q"].dtype)
    return out


def _plain_write(s):
    case, page = s["case"], s["case"]["page"]
    at = s["starts"].long()[:, None] + torch.arange(case["T"], device="cuda")
    pages, at = torch.gather(s["table"].long(), 1, at // page), at % page  # [B, T]
    kb, ks, vb, vs = _views(s["cache"], case["d"])
    (kc, kn), (vc, vn) = (_quantised(s[n].float().transpose(1, 2)) for n in ("k", "v"))
    kb[pages, :, at], ks[pages, :, at] = kc[..., 0::2] | (kc[..., 1::2] << 4), kn
    vb[pages, :, at // 4, :, at % 4] = (vc[..., 0::2] | (vc[..., 1::2] << 4)).unflatten(-1, (16, -1))
    vs[pages, :, at // 4, :, at % 4] = vn
    k = _values(_nibbles(kb[pages, :, at]), ks[pages, :, at])
    v = _values(_nibbles(vb[pages, :, at // 4, :, at % 4]).flatten(-2), vs[pages, :, at // 4, :, at % 4])
    return {"k": k.transpose(1, 2).to(s["k"].dtype), "v": v.transpose(1, 2).to(s["v"].dtype)}


def _plain_cached(s):
    case, d, page = s["case"], s["case"]["d"], s["case"]["page"]
    q = s["q"].float()
    B, H, T, _ = q.shape
    Hkv = case["Hkv"]
    k, v = (t.transpose(1, 2).flatten(2, 3) for t in
            _unpacked(s["cache"][s["table"].long().clamp(min=0)], d))  # [B, Hkv, L, d]
    q = q.reshape(B, Hkv, -1, d)
    n = s["lengths"].reshape(B, 1, 1)
    i = (n - T + torch.arange(T, device="cuda")[:, None]).repeat(1, H // Hkv, 1)[:, None]
    j = torch.arange(k.shape[2], device="cuda")
    see = (j <= i) & (i >= 0)
    if case["window"]:
        see = see & ((i - j < case["window"]) | (j < case["sinks"]))
    z = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(d))
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
    o = torch.matmul(w, v) / torch.where(total == 0, 1.0, total)
    return {"o": o.reshape(B, H, T, d).to(s["q"].dtype)}


# ---- the calls of the framework ----------------------------------------------------
def _own(s):
    import paper_2609_33591_amd as kia

    case = s["case"]
    if case["op"] == "rotary":
        plan = kia.RotaryPlan(s["freq"], layout=case["layout"], factor=s["factor"])
        out = dict(zip(("q", "k"), kia.rotary(s["q"], s["k"], plan, s["positions"])))
        if case["grad"]:
            out.update(zip(("dq", "dk"), kia.rotary(s["dq"], s["dk"], plan, s["positions"], back=True)))
        return out
    if case["op"] == "window":
        a = (case["window"], case["sinks"], s["lengths"])
        o, lse = kia.window_forward(s["q"], s["k"], s["v"], *a)
        out = {"o": o, "lse": lse}
        if case["grad"]:
            out.update(zip(("dq", "dk", "dv"),
                           kia.window_backward(s["q"], s["k"], s["v"], o, s["dO"], lse, *a)))
        return out
    cache = kia.Cache4(s["cache"], case["d"])
    if case["op"] == "write":
        kia.cache4_write(s["k"], s["v"], cache, s["table"], s["starts"])
        return dict(zip(("k", "v"), kia.cache4_read(cache, s["table"], s["starts"], case["T"], s["k"].dtype)))
    return {"o": kia.cache4_attention(s["q"], cache, s["table"], s["lengths"], K=case["K"],
                                      calib=case["calib"], tau=case["tau"], recon=case["recon"],
                                      window=case["window"], sinks=case["sinks"])}


def run(s):
    if own:
        return _own(s)
    op = s["case"]["op"]
    if op == "rotary":
        out = {"q": _plain_rotary(s["q"], s, False), "k": _plain_rotary(s["k"], s, False)}
        if s["case"]["grad"]:
            out.update(dq=_plain_rotary(s["dq"], s, True), dk=_plain_rotary(s["dk"], s, True))
        return out
    return {"window": _plain_window, "write": _plain_write, "cached": _plain_cached}[op](s)


def _seen(case):
    """(query, key) pairs that a head of each sequence takes, and the keys that any does."""
    pairs, keys, T = [], [], case["T"]
    for n in _lengths(case):
        W = case["window"] or n + 1
        at = range(n) if case["op"] == "window" else range(max(0, n - T), n)
        pairs.append(sum(min(i + 1, W) + max(0, min(case["sinks"], i + 1 - W)) for i in at))
        low = max(0, at.start + 1 - W) if len(at) else n
        keys.append(n - low + min(case["sinks"], low))
    return pairs, keys


def work(case):
    i, d = (4 if case["dtype"] == "f32" else 2), case["d"]
    if case["op"] == "rotary":
        n = case["B"] * (case["H"] + case["Hkv"]) * case["T"] * d * (2 if case["grad"] else 1)
        return {"bytes": 2 * i * n, "flops": 3 * n * case["rot"] // d}
    if case["op"] == "write":  # read, held, held read back, written
        n = 2 * case["B"] * case["Hkv"] * case["T"] * d
        return {"bytes": 2 * i * n + 2 * n * 17 // 32, "flops": n}
    pairs, keys = _seen(case)
    if case["op"] == "window":  # two products forward, five backward
        nq, nk = case["B"] * case["H"] * case["T"], case["B"] * case["Hkv"] * case["T"]
        n = (4 * nq + 4 * nk) * d if case["grad"] else (2 * nq + 2 * nk) * d
        return {"bytes": i * n + 4 * nq,
                "flops": (14 if case["grad"] else 4) * case["H"] * d * sum(pairs)}
    return {"bytes": 2 * case["Hkv"] * sum(keys) * d * 17 // 32
            + 2 * i * case["B"] * case["H"] * case["T"] * d,
            "flops": 4 * case["H"] * d * sum(pairs)}


# ---- 64 bits ------------------------------------------------------------------------
def _exact_rotary(x, s, back):
    """As a product of complex numbers."""
    case = s["case"]
    n, t = case["rot"] // 2, x.double()
    turn = torch.polar(torch.full_like(s["freq"], s["factor"]).expand(*s["positions"].shape, n),
                       s["positions"].double()[..., None] * s["freq"])[:, None]
    if case["layout"] == "half":
        z = torch.complex(t[..., :n], t[..., n:2 * n])
    else:
        z = torch.view_as_complex(t[..., :2 * n].reshape(*t.shape[:-1], n, 2).contiguous())
    z = z * (turn.conj() if back else turn)
    t = t.clone()
    if case["layout"] == "half":
        t[..., :n], t[..., n:2 * n] = z.real, z.imag
    else:
        t[..., 0:2 * n:2], t[..., 1:2 * n:2] = z.real, z.imag
    return t


def _exact_window(case, s):
    """Sequence by sequence and key head by key head, only the keys that exist,
    gradients by differentiation."""
    B, H, T, d = s["q"].shape
    G = H // case["Hkv"]
    x = {n: s[n].double() for n in ("q", "k", "v", "dO")}
    out = {"o": torch.zeros_like(x["q"]),
           "lse": torch.full((B, H, T), -math.inf, dtype=torch.float64, device="cuda")}
    if case["grad"]:
        out.update(dq=torch.zeros_like(x["q"]), dk=torch.zeros_like(x["k"]), dv=torch.zeros_like(x["v"]))
    for b, n in enumerate(_lengths(case)):
        for h in range(case["Hkv"] if n else 0):
            hs = slice(h * G, h * G + G)
            q, k, v = (t.detach().requires_grad_(case["grad"]) for t in
                       (x["q"][b, hs, :n], x["k"][b, h, :n], x["v"][b, h, :n]))
            back = torch.arange(n, device="cuda")[:, None] - torch.arange(n, device="cuda")
            hide = (back < 0) | ((back >= case["window"]) & (torch.arange(n, device="cuda") >= case["sinks"]))
            z = (q.reshape(G * n, d) @ k.T).reshape(G, n, n).div(math.sqrt(d)).masked_fill(hide, -math.inf)
            lse = torch.logsumexp(z, -1)
            o = (torch.exp(z - lse[..., None]).reshape(G * n, n) @ v).reshape(G, n, d)
            out["o"][b, hs, :n], out["lse"][b, hs, :n] = o.detach(), lse.detach()
            if case["grad"]:
                out["dq"][b, hs, :n], out["dk"][b, h, :n], out["dv"][b, h, :n] = \
                    torch.autograd.grad(o, (q, k, v), x["dO"][b, hs, :n])
    return out


def _exact_held(x):
    """The nearest of the 15 values at the group's scale, an even code between two."""
    g = x.double().reshape(*x.shape[:-1], -1, 32)
    top = g.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -130) / 6)) - 1
    for _ in range(3):
        e = torch.where(top > 6 * torch.exp2(e), e + 1, e)
    s = torch.exp2(e.clamp(-126, 125))
    level = torch.tensor(_LEVELS, dtype=torch.float64, device=x.device)
    off = (g.abs() / s)[..., None] - level
    odd = torch.arange(8, device=x.device) % 2
    near = level[(off.abs() + 1e-12 * odd).argmin(-1)]
    return (torch.copysign(near * s, g)).reshape(x.shape)


def _exact_cached(case, s):
    """Token by token: the row of its visible keys alone."""
    q, d, page, T = s["q"].double(), case["d"], case["page"], case["T"]
    out = torch.zeros_like(q)
    G = case["H"] // case["Hkv"]
    for b, n in enumerate(_lengths(case)):
        if not n:
            continue
        pages = s["cache"][s["table"][b, : (n + page - 1) // page].long()]
        k, v = (t.double().transpose(0, 1).flatten(1, 2) for t in _unpacked(pages, d))
        for t in range(max(0, T - n), T):
            i = n - T + t
            at = torch.arange(i + 1, device="cuda")
            if case["window"]:
                at = at[(at > i - case["window"]) | (at < case["sinks"])]
            z = (q[b, :, t].reshape(-1, G, d) @ k[:, at].transpose(1, 2)) / math.sqrt(d)
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
            out[b, :, t] = ((w / w.sum(-1, keepdim=True)) @ v[:, at]).reshape(-1, d)
    return {"o": out}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        out = {"q": _exact_rotary(s["q"], s, False), "k": _exact_rotary(s["k"], s, False)}
        if case["grad"]:
            out.update(dq=_exact_rotary(s["dq"], s, True), dk=_exact_rotary(s["dk"], s, True))
        return out
    if case["op"] == "window":
        return _exact_window(case, s)
    if case["op"] == "write":
        return {"k": _exact_held(s["k"]), "v": _exact_held(s["v"])}
    return _exact_cached(case, s)
