"""Host-side checks of the operators that serve from the 4-bit cache (no GPU needed): every
bad argument is refused before any launch, by the C ABI and by the binding."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import paper_2609_33591_amd as kia  # noqa: E402
from paper_2609_33591_amd.around import View  # noqa: E402

NULL, SHAPE, HEADDIM, K_, ENUM, TAU, ALIGN, HEADS, VIEW, CACHE = -1, -2, -3, -4, -5, -6, -7, -10, -11, -12
P = 4096  # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    return kia.load()


def view(B=1, H=2, T=8, d=64, data=P, **kw):
    v = dict(sb=H * T * d, sh=T * d, st=d)
    v.update(kw)
    return ctypes.byref(View(data, v["sb"], v["sh"], v["st"]))


def call(lib, op, x=None, at=0, data=P, bounds=P, pages=4, page=16, table=P, width=4, starts=P, counts=None, ws=P,
         lst=P, count=3, first=1, last=1, shared=32, freq=P, layout=0, rot=64, B=1, H=2, Hkv=2, T=8, d=64, K=4,
         calib=1, tau=8.0, recon=1, dtype=1):
    v = [view() for _ in range(4)]
    if x is not None:
        v[at] = x if x != "none" else None
    where = (pages, page, table, width)
    tail = (ws, B, H, Hkv, T, d, K, calib, tau, recon, dtype, None)
    if op == "append":
        return lib.kia_cache4_append(*v, data, bounds, *where, starts, counts, freq, 1.0, layout, B, H, Hkv, T, d,
                                     rot, dtype, None)
    if op == "bounds":
        return lib.kia_cache4_bounds(data, bounds, *where, starts, counts, B, Hkv, d, None)
    if op == "select":
        return lib.kia_cache4_select(v[0], bounds, *where, starts, ws, lst, count, first, last, B, H, Hkv, T, d,
                                     dtype, None)
    if op == "pages":
        return lib.kia_cache4_attn_pages(*v[:2], data, *where, starts, lst, count, *tail)
    return lib.kia_cache4_attn_shared(*v[:2], data, *where, starts, shared, *tail)


@pytest.mark.parametrize("op", ("append", "bounds", "select", "pages", "shared"))
def test_arguments(lib, op):
    base = dict(counts=P) if op == "bounds" else {}
    views = {"append": 4, "bounds": 0, "select": 1, "pages": 2, "shared": 2}[op]
    for kw, code in ((dict(B=0), SHAPE), (dict(Hkv=0), SHAPE), (dict(d=16), HEADDIM), (dict(d=256), HEADDIM),
                     (dict(page=48), CACHE), (dict(page=512), CACHE), (dict(pages=0), SHAPE),
                     (dict(width=0), SHAPE), (dict(width=1 << 27), SHAPE), (dict(table=None), NULL),
                     (dict(starts=None), NULL), (dict(table=P + 2), ALIGN), (dict(starts=P + 1), ALIGN)):
        assert call(lib, op, **{**base, **kw}) == code, kw
    at = "bounds" if op == "select" else "data"
    assert call(lib, op, **{**base, at: None}) == NULL
    assert call(lib, op, **{**base, at: P + 8}) == ALIGN
    for i in range(views):
        for x, code in (("none", NULL), (view(data=None), NULL), (view(data=P + 2), ALIGN), (view(st=8), VIEW),
                        (view(sh=9), VIEW), (view(st=(1 << 22) + 8), VIEW)):
            assert call(lib, op, x, i) == code, (i, code)
    if views:
        assert call(lib, op, T=0) == SHAPE and call(lib, op, dtype=7) == ENUM
    if op in ("select", "pages", "shared"):
        for kw, code in ((dict(H=3), HEADS), (dict(ws=None), NULL), (dict(ws=P + 64), ALIGN)):
            assert call(lib, op, **kw) == code, kw
    if op in ("select", "pages"):
        for kw, code in ((dict(lst=None), NULL), (dict(lst=P + 2), ALIGN), (dict(count=0), SHAPE)):
            assert call(lib, op, **kw) == code, kw
    if op in ("pages", "shared"):
        for kw, code in ((dict(K=0), K_), (dict(K=65), K_), (dict(calib=3), ENUM), (dict(recon=3), ENUM),
                         (dict(tau=0.0), TAU), (dict(tau=float("nan")), TAU),
                         (dict(B=1 << 20, H=16, Hkv=16, T=1), SHAPE)):
            assert call(lib, op, **kw) == code, kw
        # softmax looks at none of K, calib and tau: the NULL lengths stop this
        assert call(lib, op, recon=2, K=0, calib=9, tau=-1.0, starts=None) == NULL


def test_own_arguments(lib):
    for kw, code in ((dict(rot=0), HEADDIM), (dict(rot=7), HEADDIM), (dict(rot=66), HEADDIM), (dict(layout=2), ENUM),
                     (dict(freq=None), NULL), (dict(freq=P + 4), ALIGN), (dict(counts=P + 2), ALIGN),
                     (dict(bounds=P + 8), ALIGN), (dict(T=(1 << 24) + 1), SHAPE), (dict(H=65536), SHAPE),
                     (dict(B=1 << 24, T=1), SHAPE)):
        assert call(lib, "append", **kw) == code, kw
    assert call(lib, "bounds", counts=None) == NULL and call(lib, "bounds", counts=P + 1) == ALIGN
    assert call(lib, "bounds", counts=P, bounds=None) == NULL and call(lib, "bounds", counts=P, bounds=P + 4) == ALIGN
    assert call(lib, "bounds", counts=P, B=1 << 23) == SHAPE
    for kw in (dict(first=-1), dict(last=0), dict(count=2, first=2, last=1), dict(first=2147483647, last=2147483647),
               dict(H=1024, Hkv=1, d=64), dict(B=1 << 22, Hkv=4, H=4)):
        assert call(lib, "select", **kw) == SHAPE, kw
    for kw in (dict(count=200001), dict(count=1 << 28, page=256), dict(count=-5)):
        assert call(lib, "pages", **kw) == SHAPE, kw
    for kw in (dict(shared=0), dict(shared=16), dict(shared=-32), dict(shared=48), dict(shared=96),
               dict(shared=64, page=128)):
        assert call(lib, "shared", **kw) == SHAPE, kw


def test_workspaces(lib):
    n = ctypes.c_size_t(7)
    for fn, args in ((lib.kia_cache4_select_ws_bytes, (16, 4)), (lib.kia_cache4_pages_ws_bytes, (16, 4, 3)),
                     (lib.kia_cache4_shared_ws_bytes, (16, 4, 32))):
        assert fn(*args, 2, 4, 2, 3, 64, ctypes.byref(n)) == 0 and n.value > 0
        assert fn(*args, 2, 3, 2, 3, 64, ctypes.byref(n)) == HEADS and n.value == 0
        assert fn(*args, 2, 4, 2, 3, 48, ctypes.byref(n)) == HEADDIM
        assert fn(24, *args[1:], 2, 4, 2, 3, 64, ctypes.byref(n)) == CACHE
        assert fn(16, 0, *args[2:], 2, 4, 2, 3, 64, ctypes.byref(n)) == SHAPE
        assert fn(*args, 2, 4, 2, 3, 64, None) == NULL
    # every size that the checks let through: parts within their limits, no overflow
    for page in (16, 256):
        for B, H, Hkv, T in ((1, 1, 1, 1), (1, 64, 8, 1), (300, 16, 4, 5), (2, 128, 1, 40)):
            for d in (32, 128):
                for width in (1, 50, 5000, 1 << 20):
                    for count in (1, 1000, 1001, 200000):
                        rc = lib.kia_cache4_pages_ws_bytes(page, width, count, B, H, Hkv, T, d, ctypes.byref(n))
                        assert rc == 0 and n.value >= (4 + d) * 4 * B * T * H
                    for shared in (256, 4096, 1 << 24):
                        rc = lib.kia_cache4_shared_ws_bytes(page, width, shared, B, H, Hkv, T, d, ctypes.byref(n))
                        assert rc == (0 if shared <= width * page else SHAPE)
                        assert rc or n.value >= 2 * (4 + d) * 4 * B * T * H


def refuses(text, fn, *args, **kw):
    with pytest.raises(kia.KiaError, match=text):
        fn(*args, **kw)


def test_binding_refusals():
    q, k = torch.zeros(2, 4, 1, 64), torch.zeros(2, 2, 1, 64)
    cache = kia.new_cache4(3, 2, 16, 64, device="cpu")
    table, n = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    plan, bounds = kia.rotary_plan(64, device="cpu"), kia.new_bounds4(cache)
    assert bounds.shape == (3, 2, 2, 64) and bounds.dtype == torch.bfloat16 and not bounds.any()
    # append
    refuses("device tensors", kia.cache4_append, q, k, k, cache, table, n, plan)
    refuses("forward only", kia.cache4_append, q, k.clone().requires_grad_(), k, cache, table, n, plan)
    refuses("bounds must be", kia.cache4_append, q, k, k, cache, table, n, plan, bounds=bounds.float())
    refuses("bounds must be", kia.cache4_append, q, k, k, cache, table, n, plan, bounds=bounds[:2])
    refuses("starts must be", kia.cache4_append, q, k, k, cache, table, None, plan)
    refuses("counts must be", kia.cache4_append, q, k, k, cache, table, n, plan, n.long())
    refuses("has shape", kia.cache4_append, q[:1], k, k, cache, table, n, plan)
    refuses("holds 2 heads", kia.cache4_append, q, q, q, cache, table, n, plan)
    refuses("frequencies", kia.cache4_append, q, k, k, cache, table, n, kia.rotary_plan(128, device="cpu"))
    refuses("layout must be", kia.cache4_append, q, k, k, cache, table, n, kia.RotaryPlan(plan.freq, "odd"))
    refuses("device tensors", kia.cache4_bounds, cache, bounds, table, n, n)
    refuses("starts and ends", kia.cache4_bounds, cache, bounds, table, n, None)
    refuses("bounds must be", kia.cache4_bounds, cache, None, table, n, n)
    # selection
    refuses("device tensors", kia.cache4_select, q, cache, bounds, table, n, 4)
    for kw in (dict(count=0), dict(count=2.0), dict(count=4, first=-1), dict(count=4, last=0),
               dict(count=4, first=2, last=3)):
        refuses("must be", kia.cache4_select, q, cache, bounds, table, n, **kw)
    # attention
    pages = torch.zeros(2, 2, 1, 3, dtype=torch.int32)
    with torch.no_grad():
        refuses("device tensors", kia.cache4_attention, q, cache, table, n, pages=pages)
        refuses("device tensors", kia.cache4_attention, q, cache, table, n, shared=32)
        refuses("taken together", kia.cache4_attention, q, cache, table, n, pages=pages, shared=32)
        refuses("window", kia.cache4_attention, q, cache, table, n, pages=pages, window=4)
        refuses("window", kia.cache4_attention, q, cache, table, n, shared=32, sinks=4)
        refuses("pages must be", kia.cache4_attention, q, cache, table, n, pages=pages.long())
        refuses("pages must be", kia.cache4_attention, q, cache, table, n, pages=pages[0])
        refuses("pages has shape", kia.cache4_attention, q, cache, table, n, pages=pages[:, :1])
        refuses("contiguous", kia.cache4_attention, q, cache, table, n,
                pages=torch.zeros(2, 2, 1, 6, dtype=torch.int32)[..., ::2])
        refuses("multiple of 32", kia.cache4_attention, q, cache, table, n, shared=16)
        refuses("shared must be", kia.cache4_attention, q, cache, table, n, shared=-32)
        refuses("passes the table", kia.cache4_attention, q, cache, table, n, shared=96)
    refuses("forward only", kia.cache4_attention, q.clone().requires_grad_(), cache, table, n, shared=32)
