"""Host-side checks of the operators around the attention (no GPU needed): every bad
argument is refused before any launch, by the C ABI and by the binding."""
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


def rotary(lib, q=0, q_out=0, k=0, k_out=0, pos=P, sb=8, first=0, freq=P, layout=0, back=0, B=1, H=2,
           Hkv=2, T=8, d=64, rot=64, dtype=1):
    v = [view() if x == 0 else x for x in (q, q_out, k, k_out)]
    return lib.kia_rotary(*v, pos, sb, first, freq, 1.0, layout, back, B, H, Hkv, T, d, rot, dtype, None)


def test_rotary_arguments(lib):
    for kw, code in ((dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(H=0), SHAPE), (dict(Hkv=0), SHAPE),
                     (dict(d=48), HEADDIM), (dict(rot=0), HEADDIM), (dict(rot=7), HEADDIM),
                     (dict(rot=66), HEADDIM), (dict(layout=2), ENUM), (dict(back=2), ENUM),
                     (dict(dtype=2), ENUM), (dict(freq=None), NULL), (dict(q=None), NULL),
                     (dict(k=None), NULL), (dict(k_out=None), NULL), (dict(freq=P + 4), ALIGN),
                     (dict(pos=P + 2), ALIGN), (dict(sb=-1), SHAPE), (dict(first=2147483647), SHAPE),
                     (dict(q=view(data=P + 8)), ALIGN), (dict(q=view(st=60)), VIEW),
                     (dict(q=view(st=68)), VIEW), (dict(k_out=view(sh=-64)), VIEW),
                     (dict(q_out=view(st=(1 << 22) + 8)), VIEW), (dict(q=view(data=None)), NULL)):
        assert rotary(lib, **kw) == code, kw


def window(lib, fwd, x=None, at=0, lse=P, ws=P, lengths=None, B=1, H=2, Hkv=2, T=8, d=64, win=4, sinks=0,
           dtype=1):
    v = [view(T=T) for _ in range(4 if fwd else 8)]
    if x is not None:
        v[at] = x
    tail = (B, H, Hkv, T, d, win, sinks, dtype, None)
    if fwd:
        return lib.kia_window_fwd(*v, lse, lengths, *tail)
    return lib.kia_window_bwd(*v[:5], lse, lengths, ws, *v[5:], *tail)


@pytest.mark.parametrize("fwd", (True, False))
def test_window_arguments(lib, fwd):
    for kw, code in ((dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(win=0), SHAPE), (dict(sinks=-1), SHAPE),
                     (dict(H=3), HEADS), (dict(H=2, Hkv=3), HEADS), (dict(d=256), HEADDIM),
                     (dict(dtype=-1), ENUM), (dict(lse=None), NULL), (dict(lse=P + 4), ALIGN),
                     (dict(lengths=P + 1), ALIGN), (dict(T=(1 << 24) + 1), SHAPE),
                     (dict(B=1 << 20, H=1 << 10, Hkv=1, T=64), SHAPE)):
        assert window(lib, fwd, **kw) == code, kw
    for at in range(4 if fwd else 8):
        assert window(lib, fwd, ctypes.byref(View(None, 0, 0, 64)), at) == NULL
        assert window(lib, fwd, view(data=P + 2), at) == ALIGN
        assert window(lib, fwd, view(st=4), at) == VIEW
        assert window(lib, fwd, view(sh=9), at) == VIEW
    if not fwd:
        assert window(lib, fwd, ws=None) == NULL
        assert window(lib, fwd, ws=P + 16) == ALIGN
    n = ctypes.c_size_t(7)
    assert lib.kia_window_ws_bytes(1, 3, 2, 8, 64, 4, 0, ctypes.byref(n)) == HEADS and n.value == 0
    assert lib.kia_window_ws_bytes(1, 2, 2, 8, 64, 0, 0, ctypes.byref(n)) == SHAPE
    assert lib.kia_window_ws_bytes(1, 2, 2, 8, 64, 4, 0, None) == NULL
    assert lib.kia_window_ws_bytes(2, 4, 2, 100, 64, 4, 0, ctypes.byref(n)) == 0 and n.value >= 3200


def cache(lib, op, v=0, data=P, pages=4, page=16, table=P, width=4, starts=P, counts=None, ws=P, B=1, H=2,
          Hkv=2, T=8, d=64, K=4, calib=1, tau=8.0, recon=1, win=0, sinks=0, dtype=1):
    a = view() if v == 0 else v
    if op == "attn":
        return lib.kia_cache4_attn(a, view(), data, pages, page, table, width, starts, ws, B, H, Hkv, T, d,
                                   K, calib, tau, recon, win, sinks, dtype, None)
    tail = (B, Hkv, T, d, dtype, None)
    if op == "write":
        return lib.kia_cache4_write(a, view(), data, pages, page, table, width, starts, counts, *tail)
    return lib.kia_cache4_read(data, pages, page, table, width, starts, counts, a, view(), *tail)


@pytest.mark.parametrize("op", ("write", "read", "attn"))
def test_cache_arguments(lib, op):
    for kw, code in ((dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(d=16), HEADDIM), (dict(page=48), CACHE),
                     (dict(page=512), CACHE), (dict(page=8), CACHE), (dict(pages=0), SHAPE),
                     (dict(width=0), SHAPE), (dict(width=1 << 27), SHAPE), (dict(dtype=7), ENUM),
                     (dict(data=None), NULL), (dict(table=None), NULL), (dict(starts=None), NULL),
                     (dict(v=None), NULL), (dict(data=P + 8), ALIGN), (dict(table=P + 2), ALIGN),
                     (dict(starts=P + 1), ALIGN), (dict(v=view(st=8)), VIEW)):
        assert cache(lib, op, **kw) == code, kw
    if op != "attn":
        assert cache(lib, op, counts=P + 2) == ALIGN
        return
    for kw, code in ((dict(H=3), HEADS), (dict(K=0), K_), (dict(K=65), K_), (dict(calib=3), ENUM),
                     (dict(recon=3), ENUM), (dict(recon=-1), ENUM), (dict(tau=0.0), TAU),
                     (dict(tau=float("nan")), TAU), (dict(calib=2, tau=float("inf")), TAU),
                     (dict(win=-1), SHAPE), (dict(sinks=-1), SHAPE), (dict(ws=None), NULL),
                     (dict(ws=P + 64), ALIGN)):
        assert cache(lib, op, **kw) == code, kw
    # softmax looks at none of K, calib and tau, MinMax not at tau: the NULL lengths stop these
    assert cache(lib, op, recon=2, K=0, calib=9, tau=-1.0, starts=None) == NULL
    assert cache(lib, op, calib=0, tau=-1.0, starts=None) == NULL
    n = ctypes.c_size_t(7)
    assert lib.kia_cache4_bytes(4, 16, 2, 64, ctypes.byref(n)) == 0 and n.value == 4 * 2 * 2 * 16 * 34
    assert lib.kia_cache4_bytes(4, 24, 2, 64, ctypes.byref(n)) == CACHE and n.value == 0
    assert lib.kia_cache4_bytes(0, 16, 2, 64, ctypes.byref(n)) == SHAPE
    assert lib.kia_cache4_ws_bytes(16, 4, 1, 3, 2, 1, 64, 0, 0, ctypes.byref(n)) == HEADS


def test_error_texts():
    for code in (HEADS, VIEW, CACHE):
        assert kia.kia_strerror(code) != "unknown error code"


def refuses(text, fn, *args, **kw):
    with pytest.raises(kia.KiaError, match=text):
        fn(*args, **kw)


def test_binding_refusals():
    q = torch.zeros(2, 4, 8, 64)
    k = torch.zeros(2, 2, 8, 64)
    refuses("device tensors", kia.window_forward, q, k, k, 4)
    refuses("window must be", kia.window_forward, q, k, k, 0)
    refuses("window must be", kia.window_forward, q, k, k, 4.0)
    refuses("sinks must be", kia.window_forward, q, k, k, 4, -1)
    refuses("lengths must be", kia.window_forward, q, k, k, 4, 0, [8, 8])
    refuses("lengths must be", kia.window_forward, q, k, k, 4, 0, torch.zeros(2))
    refuses("lengths has shape", kia.window_forward, q, k, k, 4, 0, torch.zeros(3, dtype=torch.int32))
    refuses("positions without", kia.window_attention, q, k, k, 4, positions=3)
    plan = kia.rotary_plan(64, device="cpu")
    refuses("device tensors", kia.rotary, q, k, plan)
    for kw in (dict(rot=63), dict(rot=0), dict(rot=64, layout="odd"), dict(rot=64, scaling="odd"),
               dict(rot=64, base=0.0), dict(rot=64, scaling="parts"), dict(rot=64, stretch=0.0)):
        with pytest.raises(kia.KiaError):
            kia.rotary_plan(**kw, device="cpu")
    refuses("heads of 32, 64 or 128", kia.Cache4, torch.zeros(1, 2, 1, 16 * 34, dtype=torch.uint8), 48)
    refuses("no cache of heads", kia.Cache4, torch.zeros(1, 2, 1, 24 * 34, dtype=torch.uint8), 64)
    refuses("uint8", kia.Cache4, torch.zeros(1, 2, 1, 16 * 34), 64)
    refuses("uint8", kia.Cache4, torch.zeros(1, 1, 1, 16 * 34, dtype=torch.uint8), 64)
    cache = kia.new_cache4(3, 2, 16, 64, device="cpu")
    assert (cache.pages, cache.heads, cache.page, cache.d) == (3, 2, 16, 64) and not cache.data.any()
    refuses("page must be", kia.new_cache4, 3, 2, 48, 64, device="cpu")
    table, one = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    refuses("device tensors", kia.cache4_write, k, k, cache, table, one)
    refuses("forward only", kia.cache4_attention, q.requires_grad_(), cache, table, one)
    refuses("holds heads of 64", kia.cache4_attention, torch.zeros(2, 4, 1, 32), cache, table, one)
    refuses("table must be", kia.cache4_attention, q.detach(), cache, table.long(), one)
    refuses("window must be", kia.cache4_attention, q.detach(), cache, table, one, window=-1)


def test_view_checks_without_a_device():
    """Layouts that the kernels cannot take are found (and copied by the allocating calls)."""
    from paper_2609_33591_amd.around import _Like
    x = torch.zeros(2, 8, 4, 64)
    for y in (x, x.transpose(1, 2), x[:1].expand(2, 8, 4, 64)):
        like = _Like("y", y)
        assert like.take("y", y)[0] is y
        v = like.view("y", y)
        assert (v.data, v.sb, v.sh, v.st) == (y.data_ptr(), *y.stride()[:3])
    for y in (x.transpose(2, 3), torch.zeros(2, 8, 4, 65)[..., :64], torch.zeros(2, 8, 4, 66)[..., 2:],
              x[:, :, :1].expand(2, 8, 4, 64)):
        like = _Like("y", y)
        refuses("y ", like.view, "y", y)
        z, v = like.take("y", y)
        assert z is not y and torch.equal(z, y) and v.data == z.data_ptr()
    y = torch.arange(2 * 8 * 4 * 64 + 1.0)[1:].view(2, 8, 4, 64)  # contiguous, 4 bytes off
    assert y.is_contiguous() and _Like("y", y).take("y", y)[0] is not y
    refuses("must not be expanded", _Like("x", x).view, "x", x[:1].expand(2, 8, 4, 64), None, True)
