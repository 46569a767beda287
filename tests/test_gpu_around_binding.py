"""The binding's two ways of the same calls: in C where every argument is as the kernels
take it, in Python with copies otherwise. Same bits, same errors, nothing leaked."""
import gc
import sys

import pytest

torch = pytest.importorskip("torch")

import paper_2609_33591_amd as kia  # noqa: E402
from paper_2609_33591_amd import around  # noqa: E402

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


def calls(dtype):
    g = torch.Generator().manual_seed(1)
    q, k, v, dO = (torch.randn(2, h, 40, 64, generator=g).to(dtype).cuda() for h in (4, 2, 2, 4))
    plan = kia.rotary_plan(32)
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    n = torch.tensor([40, 7], dtype=torch.int32, device="cuda")
    cache = kia.new_cache4(8, 2, 16, 64)
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3)
    zero = torch.zeros_like(n)
    return {
        "rotary": lambda: kia.rotary(q, k, plan, pos),
        "rotary2": lambda: kia.rotary(q, None, plan, pos.expand(2, 40).contiguous(), back=True)[:1],
        "rotary3": lambda: kia.rotary(q.transpose(1, 2).contiguous().transpose(1, 2), k, plan, -5),
        "forward": lambda: kia.window_forward(q, k, v, 9, 2, n),
        "backward": lambda: kia.window_backward(q, k, v, *kia.window_forward(q, k, v, 9, 2)[:1], dO,
                                                kia.window_forward(q, k, v, 9, 2)[1], 9, 2),
        "cache": lambda: (kia.cache4_write(k, v, cache, table, zero, n),
                          *kia.cache4_read(cache, table, zero, 40, dtype))[1:],
        "attention": lambda: (kia.cache4_attention(q, cache, table, n, recon="softmax", window=5, sinks=1),
                              kia.cache4_attention(q, cache, table, n)),
    }


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("name", ("rotary", "rotary2", "rotary3", "forward", "backward", "cache", "attention"))
def test_same_results(both, dtype, name):
    fast, slow = both(calls(dtype)[name])
    assert len(fast) == len(slow)
    for a, b in zip(fast, slow):
        assert a.shape == b.shape and a.dtype == b.dtype and a.stride() == b.stride()
        assert torch.equal(a, b)


def test_same_errors(both):
    q = torch.zeros(1, 4, 8, 64, device="cuda")
    k = torch.zeros(1, 2, 8, 64, device="cuda")
    n = torch.zeros(1, dtype=torch.int32, device="cuda")
    table = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    cache, plan = kia.new_cache4(2, 2, 16, 64), kia.rotary_plan(64)
    odd = torch.zeros(1, 3, 8, 64, device="cuda")
    for fn in (lambda: kia.window_forward(q, odd, odd, 4), lambda: kia.window_forward(q, k, k.bfloat16(), 4),
               lambda: kia.window_forward(q, k, k, True), lambda: kia.window_forward(q, k, k, 4, 0, n.long()),
               lambda: kia.window_forward(q.half(), k.half(), k.half(), 4),
               lambda: kia.window_forward(q[0], k, k, 4), lambda: kia.window_forward(q, k, k, 1 << 31),
               lambda: kia.window_forward(q.cpu(), k.cpu(), k.cpu(), 4),
               lambda: kia.window_forward(torch.zeros(1, 2, 8, 48, device="cuda"), *[odd[..., :48].contiguous()[:, :1]] * 2, 4),
               lambda: kia.window_backward(q, k, k, q, q, torch.zeros(1, 4, 7, device="cuda"), 4),
               lambda: kia.rotary(q, k, kia.RotaryPlan(plan.freq.float())),
               lambda: kia.rotary(q, k, kia.RotaryPlan(plan.freq, "odd")),
               lambda: kia.rotary(q, k, kia.RotaryPlan(plan.freq.repeat(2))),
               lambda: kia.rotary(q, k, plan, torch.zeros(7, dtype=torch.int32, device="cuda")),
               lambda: kia.rotary(q, k, plan, 2.0),
               lambda: kia.cache4_write(k, k, cache, table, None), lambda: kia.cache4_write(q, q, cache, table, n),
               lambda: kia.cache4_attention(odd, cache, table, n), lambda: kia.cache4_attention(q, cache, table.long(), n),
               lambda: kia.cache4_attention(q, cache, table, n, K=0),
               lambda: kia.cache4_attention(q, cache, table, n, tau=float("nan")),
               lambda: kia.cache4_attention(q, cache, table, n, recon="bf16_exp"),
               lambda: kia.cache4_read(cache, table, n, 0, torch.float32)):
        def text():
            with pytest.raises(kia.KiaError) as e:
                fn()
            return str(e.value)
        fast, slow = both(text)
        assert fast == slow


def test_nothing_is_kept():
    """Reference counts of the arguments, and the memory of the results, are given back."""
    every = calls(torch.bfloat16)
    for fn in every.values():
        fn()
    gc.collect()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    counts = [sys.getrefcount(x) for x in (None, torch.float32, torch.uint8, torch.Tensor)]
    for fn in every.values():
        for _ in range(200):
            fn()
    gc.collect()
    assert torch.cuda.memory_allocated() == before
    after = [sys.getrefcount(x) for x in (None, torch.float32, torch.uint8, torch.Tensor)]
    assert all(abs(a - b) < 100 for a, b in zip(after, counts))
