"""The operators that serve many and long texts from the 4-bit cache, from their
definitions in 64 bits, and the caches that their tests use."""
import math

import torch

import paper_2609_33591_amd as kia
from tests import around_reference as ref


def draw(shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def table_of(lengths, page, seed, shared=0, spare=2, width=None):
    """Pages in random order, the first `shared` tokens' the same ones for all, and how many
    there are."""
    common = shared // page
    need = [max(0, (n + page - 1) // page - common) for n in lengths]
    total = common + sum(need) + spare
    order = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).tolist()
    t = torch.full((len(lengths), width or max(1, common + max(need))), -1, dtype=torch.int32)
    for i in range(common):
        t[:, i] = order.pop()
    for b, n in enumerate(need):
        for i in range(n):
            t[b, common + i] = order.pop()
    return t.cuda(), total


def filled(lengths, Hkv, d, page, dtype, seed, scale=0.7, shared=0, change=None, width=None):
    """A cache of random tokens behind `shared` common ones, its table, its bounds, and the
    values it stands for, [B, Hkv, T, d]."""
    table, pages = table_of(lengths, page, seed, shared, width=width)
    cache = kia.new_cache4(pages, Hkv, page, d)
    T = max(max(lengths), 1)
    k, v = draw((len(lengths), Hkv, T, d), dtype, seed + 1, scale), draw((len(lengths), Hkv, T, d), dtype, seed + 2)
    k[..., ::16] *= 3
    k += draw((len(lengths), Hkv, (T + page - 1) // page, d), dtype, seed + 3, scale).repeat_interleave(page, 2)[:, :, :T]
    k[:, :, :shared], v[:, :, :shared] = k[:1, :, :shared], v[:1, :, :shared]
    if change:
        change(k, v)
    n = ints(*lengths)
    zero = torch.zeros_like(n)
    kia.cache4_write(k, v, cache, table, zero, n)
    bounds = kia.new_bounds4(cache)
    kia.cache4_bounds(cache, bounds, table, zero, n)
    return cache, table, bounds, ref.held(k), ref.held(v)


def bounds_of(held, n, page, w):
    """Bounds [Hkv, 2, d] of page w of keys held [Hkv, T, d], of which n count; NaN stays."""
    x = held[:, w * page:min(n, w * page + page)]
    return torch.stack((x.amin(1), x.amax(1)), 1)


def select(q, bounds, table, n, page, pages, count, first, last):
    """Pages of q [H, T, d] (the last of n tokens) by bounds [W, Hkv, 2, d] in the order of
    the table; list [Hkv][T]."""
    H, T, d = q.shape
    Hkv = bounds.shape[1]
    G, q = H // Hkv, q.double()
    out = []
    for h in range(Hkv):
        out.append([])
        for t in range(T):
            i = n - T + t
            ws = [w for w in range(i // page + 1) if 0 <= table[w] < pages] if i >= 0 else []
            if len(ws) > count:
                lo, hi = bounds[ws, h].double().unbind(1)
                x = q[h * G:h * G + G, t, None]
                s = torch.where(x > 0, x * hi, x * lo).sum(-1).nan_to_num(nan=math.inf, posinf=math.inf, neginf=-math.inf)
                s = dict(zip(ws, s.amax(0).tolist()))
                must = {w for w in ws if w < first or w > i // page - last}
                rest = sorted((w for w in ws if w not in must), key=lambda w: (-s[w], w))
                ws = sorted(must) + rest[:count - len(must)]
            out[-1].append(sorted(ws) + [-1] * (count - len(ws)))
    return out


def over_pages(q, k, v, n, page, pages, **op):
    """(value, bound) of q [H, T, d], the last of n tokens, over the listed pages
    [Hkv, T, count] of keys and values [Hkv, n, d]."""
    H, T, d = q.shape
    Hkv = k.shape[0]
    G = H // Hkv
    o, bound = torch.zeros(H, T, d, dtype=torch.float64, device=q.device), \
        torch.zeros(H, T, d, dtype=torch.float64, device=q.device)
    for h in range(Hkv):
        for t in range(T):
            i = n - T + t
            at = [j for w in pages[h][t] if w >= 0 for j in range(w * page, min(w * page + page, i + 1))]
            if not at:
                continue
            g = slice(h * G, h * G + G)
            a, b = ref.cached(q[g, t:t + 1], k[h:h + 1, at], v[h:h + 1, at], len(at), **op)
            o[g, t], bound[g, t] = a[:, 0], b[:, 0]
    return o, bound
