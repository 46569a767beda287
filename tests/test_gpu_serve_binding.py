"""The binding's two ways of the calls that serve from the 4-bit cache: in C where every
argument is as the kernels take it, in Python with copies otherwise. Same bits, same errors,
nothing leaked; and the calls on buffers of the caller's."""
import gc
import sys

import pytest

torch = pytest.importorskip("torch")

import paper_2609_33591_amd as kia  # noqa: E402
from paper_2609_33591_amd import around  # noqa: E402
from tests.serve_reference import draw, filled, ints  # noqa: E402

pytestmark = pytest.mark.gpu


class Slow:
    """The C module that takes no call."""

    def __getattr__(self, name):
        return lambda *a: None


@pytest.fixture
def both(monkeypatch):
    def run(fn):
        fast = fn()
        monkeypatch.setattr(around, "_fast", lambda: Slow())
        slow = fn()
        monkeypatch.undo()
        return fast, slow
    return run


def setting(dtype):
    lengths = (200, 130)
    cache, table, bounds, k, v = filled(lengths, 2, 64, 32, dtype, 1, 0.7, 64, width=8)
    return cache, table, bounds, draw((2, 6, 2, 64), dtype, 5), draw((2, 2, 2, 64), dtype, 6), ints(*lengths)


def calls(dtype):
    cache, table, bounds, q, k, n = setting(dtype)
    plan, odd = kia.rotary_plan(32, layout="interleaved"), torch.cat((q, q), 3)[..., 1:65]
    pages = kia.cache4_select(q, cache, bounds, table, n, 3)
    return {
        "append": lambda: (kia.cache4_append(q, k, k, cache, table, n, plan, ints(1, 2), bounds), cache.data.clone(),
                           bounds.clone()),
        "append2": lambda: (kia.cache4_append(odd, k, k, cache, table, n, plan), cache.data.clone()),
        "select": lambda: (kia.cache4_select(q, cache, bounds, table, n, 4, 0, 2),
                           kia.cache4_select(odd, cache, bounds, table, n, 4, 0, 2)),
        "pages": lambda: (kia.cache4_attention(q, cache, table, n, pages=pages, recon="softmax"),
                          kia.cache4_attention(q, cache, table, n, pages=pages, K=4)),
        "shared": lambda: (kia.cache4_attention(q, cache, table, n, shared=64, recon="softmax"),
                           kia.cache4_attention(odd, cache, table, n, shared=64)),
    }


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("name", ("append", "append2", "select", "pages", "shared"))
def test_same_results(both, dtype, name):
    fast, slow = both(calls(dtype)[name])
    assert len(fast) == len(slow)
    for a, b in zip(fast, slow):
        assert a.shape == b.shape and a.dtype == b.dtype and a.stride() == b.stride()
        assert torch.equal(a, b)


def test_same_errors(both):
    cache, table, bounds, q, k, n = setting(torch.float32)
    plan, pages = kia.rotary_plan(64), torch.zeros(2, 2, 2, 3, dtype=torch.int32, device="cuda")
    for fn in (lambda: kia.cache4_append(q, k, k, cache, table, None, plan),
               lambda: kia.cache4_append(q, k, k, cache, table, n, kia.RotaryPlan(plan.freq.float())),
               lambda: kia.cache4_append(q, k, k, cache, table, n, kia.RotaryPlan(plan.freq, "odd")),
               lambda: kia.cache4_append(q, q, q, cache, table, n, plan),
               lambda: kia.cache4_append(q.half(), k.half(), k.half(), cache, table, n, plan),
               lambda: kia.cache4_append(q, k, k, cache, table, n, plan, bounds=bounds.float()),
               lambda: kia.cache4_append(q, k, k, cache, table, n, plan, bounds=bounds[:3]),
               lambda: kia.cache4_select(q, cache, bounds, table, n.long(), 3),
               lambda: kia.cache4_select(q, cache, bounds[..., :32], table, n, 3),
               lambda: kia.cache4_select(q, cache, bounds, table, n, 1),
               lambda: kia.cache4_select(q, cache, bounds, table, n, 3, True),
               lambda: kia.cache4_select(q[:, :3], cache, bounds, table, n, 3),
               lambda: kia.cache4_attention(q, cache, table, n, pages=pages.long()),
               lambda: kia.cache4_attention(q, cache, table, n, pages=pages[:1]),
               lambda: kia.cache4_attention(q, cache, table, n, pages=pages[..., :0]),
               lambda: kia.cache4_attention(q, cache, table, n, shared=48),
               lambda: kia.cache4_attention(q, cache, table, n, shared=512),
               lambda: kia.cache4_attention(q, cache, table, n, shared=64, K=0),
               lambda: kia.cache4_attention(q[:, :3], cache, table, n, shared=64),
               lambda: kia.cache4_attention(q, cache, table, n, shared=64, recon="bf16_exp")):
        def text():
            with pytest.raises(kia.KiaError) as e:
                fn()
            return str(e.value)
        fast, slow = both(text)
        assert fast == slow


def test_buffers_of_the_callers():
    """The kia_* calls write into what they are given, on a stream of the caller's."""
    cache, table, bounds, q, k, n = setting(torch.bfloat16)
    plan, side = kia.rotary_plan(64), torch.cuda.Stream()
    want = kia.cache4_append(q, k, k, cache, table, n - 2, plan, bounds=bounds)
    pages = kia.cache4_select(want, cache, bounds, table, n, 3)
    outs = (kia.cache4_attention(want, cache, table, n, pages=pages), kia.cache4_attention(want, cache, table, n, shared=64))
    data, edges = cache.data.clone(), bounds.clone()
    torch.cuda.synchronize()
    x, o, lst = torch.empty_like(q), torch.empty_like(q), torch.empty_like(pages)
    sizes = (kia.kia_cache4_select_ws_bytes(32, 8, 2, 6, 2, 2, 64), kia.kia_cache4_pages_ws_bytes(32, 8, 3, 2, 6, 2, 2, 64),
             kia.kia_cache4_shared_ws_bytes(32, 8, 64, 2, 6, 2, 2, 64))
    ws = [torch.full((s,), 255, dtype=torch.uint8, device="cuda") for s in sizes]
    starts = n - 2
    torch.cuda.synchronize()
    kia.kia_cache4_append(q, x, k, k, cache, table, starts, plan, bounds=bounds, stream=side)
    kia.kia_cache4_bounds(cache, bounds, table, starts, n, stream=side)
    kia.kia_cache4_select(x, lst, cache, bounds, table, n, ws[0], stream=side)
    kia.kia_cache4_attn_pages(x, o, cache, table, n, lst, ws[1], stream=side)
    side.synchronize()
    assert torch.equal(x, want) and torch.equal(cache.data, data) and torch.equal(bounds, edges)
    assert torch.equal(lst, pages) and torch.equal(o, outs[0])
    kia.kia_cache4_attn_shared(x, o, cache, table, n, 64, ws[2], stream=side)
    side.synchronize()
    assert torch.equal(o, outs[1])
    for call, at in ((kia.kia_cache4_attn_pages, (lst, ws[1][:-256])), (kia.kia_cache4_attn_shared, (64, ws[2][:-256]))):
        with pytest.raises(kia.KiaError, match="ws holds"):
            call(x, o, cache, table, n, *at)
    with pytest.raises(kia.KiaError, match="ws holds"):
        kia.kia_cache4_select(x, lst, cache, bounds, table, n, ws[0][:16])


def test_nothing_is_kept():
    """Reference counts of the arguments, and the memory of the results, are given back."""
    every = calls(torch.bfloat16)
    for fn in every.values():
        fn()
    gc.collect()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    counts = [sys.getrefcount(x) for x in (None, torch.float32, torch.uint8, torch.int32, torch.Tensor)]
    for fn in every.values():
        for _ in range(200):
            fn()
    gc.collect()
    assert torch.cuda.memory_allocated() == before
    after = [sys.getrefcount(x) for x in (None, torch.float32, torch.uint8, torch.int32, torch.Tensor)]
    assert all(abs(a - b) < 100 for a, b in zip(after, counts))
