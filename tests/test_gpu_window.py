"""Softmax attention with a sliding window and visible first tokens on the device,
forward and backward, against its definition in 64 bits; every bound is derived in
around_reference.window from the roundings that the kernels are allowed."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2609_33591_amd as kia  # noqa: E402
from tests import around_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = (torch.float32, torch.bfloat16)


def draw(shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def inputs(B, H, Hkv, T, d, dtype, seed=1, scale=1.0):
    return (draw((B, H, T, d), dtype, seed, scale), draw((B, Hkv, T, d), dtype, seed + 1, scale),
            draw((B, Hkv, T, d), dtype, seed + 2), draw((B, H, T, d), dtype, seed + 3))


def check(q, k, v, g, window, sinks, lengths=None):
    want = ref.window(q, k, v, window, sinks, lengths, g)
    o, lse = kia.window_forward(q, k, v, window, sinks, lengths)
    grads = kia.window_backward(q, k, v, o, g, lse, window, sinks, lengths)
    for name, x in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *grads)):
        ref.within(x, *want[name], name)
    return o, lse, grads


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,H,Hkv,T,d,window,sinks", [
    (1, 1, 1, 1, 16, 1, 0), (1, 1, 1, 2, 32, 1, 0), (2, 2, 1, 31, 16, 5, 2), (1, 3, 3, 32, 64, 32, 0),
    (1, 2, 2, 33, 128, 1, 1), (1, 4, 2, 64, 32, 64, 0), (2, 2, 1, 65, 64, 20, 2),
    (1, 2, 2, 128, 128, 1000, 0), (1, 6, 2, 129, 64, 64, 33), (1, 2, 1, 200, 128, 70, 4),
    (1, 8, 1, 257, 32, 100, 130), (1, 1, 1, 300, 16, 2, 0), (2, 7, 7, 96, 64, 3, 96),
    (1, 4, 4, 333, 128, 129, 64), (1, 2, 1, 520, 64, 17, 1)])
def test_forward_and_backward(dtype, B, H, Hkv, T, d, window, sinks):
    check(*inputs(B, H, Hkv, T, d, dtype), window, sinks)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", (0.01, 6.0))
def test_flat_and_sharp_rows(dtype, scale):
    """Scores of almost the same size, and rows that one key takes."""
    check(*inputs(1, 2, 1, 150, 64, dtype, seed=20, scale=scale), 40, 3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", (32, 128))
def test_padded_batch(dtype, d):
    """Sequences of 0, 1, some and all tokens; NaN and infinities behind their ends
    reach nothing, and outputs there are 0."""
    B, H, Hkv, T = 5, 4, 2, 140
    lengths = torch.tensor([0, 1, 63, 140, 129], dtype=torch.int32, device="cuda")
    q, k, v, g = inputs(B, H, Hkv, T, d, dtype, seed=30)
    for x, bad in zip((q, k, v, g), (math.nan, math.inf, -math.inf, math.nan)):
        for b, n in enumerate(lengths.tolist()):
            x[b, :, n:] = bad
    o, lse, grads = check(q, k, v, g, 50, 2, lengths)
    for b, n in enumerate(lengths.tolist()):
        assert all(not x[b, :, n:].any() for x in (o, *grads))
        assert bool((lse[b, :, n:] == -math.inf).all())
    # lengths that are out of range are taken as the nearest in it
    wide = torch.tensor([-3, 1, 63, 900, 129], dtype=torch.int32, device="cuda")
    again = kia.window_forward(q, k, v, 50, 2, wide)
    assert torch.equal(again[0], o) and torch.equal(again[1], lse)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", (math.nan, math.inf, -math.inf))
def test_what_is_not_seen_has_no_influence(dtype, bad):
    """One row of k, v, q or dO with infinities or NaNs: rows that do not see it (keys
    that it does not see) are the same, bit for bit; those that do are not finite."""
    B, H, Hkv, T, d, window, sinks, at = 1, 2, 1, 150, 64, 30, 2, 77
    clean = inputs(B, H, Hkv, T, d, dtype, seed=40)
    o0, lse0, (dq0, dk0, dv0) = check(*clean, window, sinks)
    rows = torch.arange(T, device="cuda")
    see = (rows >= at) & (rows - at < window)  # queries that see key `at`
    seen = (rows <= at) & ((at - rows < window) | (rows < sinks))  # keys that query `at` sees
    for which in range(4):
        x = [t.clone() for t in clean]
        x[which][:, :, at, 5] = bad
        q, k, v, g = x
        o, lse = kia.window_forward(q, k, v, window, sinks)
        dq, dk, dv = kia.window_backward(q, k, v, o, g, lse, window, sinks)
        hit = {0: rows == at, 1: see, 2: see, 3: rows < 0}[which]
        assert torch.equal(o[:, :, ~hit], o0[:, :, ~hit])
        assert torch.equal(lse[:, :, ~hit] if which < 2 else lse, lse0[:, :, ~hit] if which < 2 else lse0)
        if which == 2:
            assert not torch.isfinite(o[:, :, see, 5]).any()
            assert torch.equal(o[..., :5], o0[..., :5]) and torch.equal(o[..., 6:], o0[..., 6:])
        rowhit = {0: rows == at, 1: see, 2: see, 3: rows == at}[which]
        assert torch.equal(dq[:, :, ~rowhit], dq0[:, :, ~rowhit])
        # keys that some hit query sees
        touched = seen if which in (0, 3) else \
            ((rows[None] <= rows[:, None]) & ((rows[:, None] - rows[None] < window) | (rows[None] < sinks)))[see].any(0)
        assert torch.equal(dk[:, :, ~touched], dk0[:, :, ~touched])
        assert torch.equal(dv[:, :, ~touched], dv0[:, :, ~touched])
        if which in (0, 3):
            assert not torch.isfinite(dk[:, :, seen]).all(-1).any()


@pytest.mark.parametrize("dtype", TYPES)
def test_views_and_outputs(dtype):
    """Heads of a fused projection, keys shared by a batch, and outputs written into a
    larger buffer, whose other rows stay as they were."""
    B, H, Hkv, T, d, window, sinks = 2, 4, 2, 90, 64, 25, 3
    qkv = draw((B, T, H + 2 * Hkv, d), dtype, 50)
    q, k, v = (x.transpose(1, 2) for x in qkv.split((H, Hkv, Hkv), 2))
    g = draw((B, T, H, d), dtype, 51).transpose(1, 2)
    o, lse, grads = check(q, k, v, g, window, sinks)
    same = check(*(x.contiguous() for x in (q, k, v, g)), window, sinks)
    assert all(torch.equal(a, b) for a, b in zip((o, lse, *grads), (same[0], same[1], *same[2])))
    shared = (k[:1].expand(B, Hkv, T, d), v[:1].expand(B, Hkv, T, d))
    check(q, *shared, g, window, sinks)
    big = torch.full((B, T + 2, H, d), 7.0, dtype=dtype, device="cuda")
    out = big[:, 1:-1].transpose(1, 2)
    kia.kia_window_fwd(q, k, v, out, lse, window, sinks)
    assert torch.equal(out, o)
    assert bool((big[:, 0] == 7).all()) and bool((big[:, -1] == 7).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_parts_of_long_key_lists(dtype):
    """First tokens that every one of many queries sees, over shared heads: their key
    block's queries are cut into parts, whose sums repeat bit for bit."""
    q, k, v, g = inputs(1, 4, 1, 1500, 32, dtype, seed=60)
    o, lse, grads = check(q, k, v, g, 130, 5)
    for _ in range(3):
        again = kia.window_backward(q, k, v, o, g, lse, 130, 5)
        assert all(torch.equal(a, b) for a, b in zip(again, grads))


def test_autograd_broadcast_inputs_and_differences():
    B, H, Hkv, T, d, window, sinks = 2, 4, 2, 40, 32, 9, 2
    q, k, v, g = inputs(B, H, Hkv, T, d, torch.float32, seed=70)
    # keys shared by the batch: their gradient is summed over it
    k1, v1 = k[:1].clone().requires_grad_(), v[:1].clone().requires_grad_()
    x = q.clone().requires_grad_()
    o = kia.window_attention(x, k1.expand_as(k), v1.expand_as(v), window, sinks)
    got = torch.autograd.grad(o, (x, k1, v1), g)
    want = ref.window(q, k[:1].expand_as(k), v[:1].expand_as(v), window, sinks, None, g)
    ref.within(got[0], *want["dq"], "dq")
    for i, n in ((1, "dk"), (2, "dv")):
        y, e = (t.sum(0, keepdim=True) for t in want[n])
        ref.within(got[i], y, e + B * ref.E * want[n][0].abs().sum(0, keepdim=True), n)
    # against differences of the loss in float64 sums: outputs of order 1 are off by
    # about 64 E each, over a step of 2^-4, and the cubic term of the step
    def loss(q, k, v):
        return (kia.window_attention(q, k, v, window, sinks).double() * g).sum().item()

    args = [q, k, v]
    o, lse = kia.window_forward(q, k, v, window, sinks)
    grads = kia.window_backward(q, k, v, o, g, lse, window, sinks)
    for i, at in ((0, (1, 3, 39, 7)), (1, (0, 1, 1, 30)), (1, (1, 0, 22, 4)), (2, (0, 0, 0, 31))):
        def slope(eps):
            moved = []
            for sign in (1, -1):
                y = [t.clone() for t in args]
                y[i][at] += sign * eps
                moved.append(loss(*y))
            return (moved[0] - moved[1]) / (2 * eps)
        # (extrapolated to a step of 0: the cubic term cancels)
        s = (4 * slope(2.0 ** -5) - slope(2.0 ** -4)) / 3
        assert abs(s - float(grads[i][at])) <= 2e-3 * (1 + abs(s))


def test_other_stream_and_capture():
    """A graph of the forward and the backward replays to the same bits, with eager
    work between; and calls on a stream of the caller's."""
    q, k, v, g = inputs(1, 4, 2, 300, 64, torch.bfloat16, seed=80)
    o, lse = kia.window_forward(q, k, v, 64, 3)
    want = (o, lse, *kia.window_backward(q, k, v, o, g, lse, 64, 3))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = kia.window_forward(q, k, v, 64, 3)
        b = kia.window_backward(q, k, v, a[0], g, a[1], 64, 3)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip((*a, *b), want))
    static = [x.clone() for x in (q, k, v, g)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a = kia.window_forward(*static[:3], 64, 3)
        b = kia.window_backward(*static[:3], a[0], static[3], a[1], 64, 3)
    for turn in range(3):
        for s, x in zip(static, (q, k, v, g)):
            s.copy_(x if turn != 1 else x.flip(2))
        graph.replay()
        torch.cuda.synchronize()
        if turn != 1:
            assert all(torch.equal(x, y) for x, y in zip((*a, *b), want))
        else:
            e = kia.window_forward(*static[:3], 64, 3)
            assert torch.equal(a[0], e[0]) and torch.equal(a[1], e[1])
