"""Calls at the edges of what the operators around the attention take, on the device:
each is compared with its definition in 64 bits, or bit for bit with the same call in
another form."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2609_33591_amd as kia  # noqa: E402
from tests import around_reference as ref  # noqa: E402
from tests.test_gpu_cache4 import TYPES, check, draw, filled, ints  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("op", (dict(recon="softmax"), dict(recon="lerp", calib="fwm", K=4, tau=8.0)),
                         ids=lambda o: o["recon"])
def test_values_of_nan_in_parts_of_no_weight(op):
    """A value of NaN under a weight that is 0 makes the rows that see it NaN, wherever
    the keys are cut into parts."""
    n, at = 4000, 3000  # (the last quarter of the keys has no weight: whole parts)

    def change(k, v):
        k[..., :at, :] = 0.5
        k[..., at:, :] = -3.0  # scores 350 below the others'
        v[..., 3990, 7] = math.nan

    cache, table, k, v = filled((n,), 1, 64, 64, torch.float32, 100, change=change)
    q = torch.full((1, 4, 2, 64), 12.5, device="cuda")
    o = kia.cache4_attention(q, cache, table, ints(n), **op)
    assert torch.isnan(o[..., :32]).all()
    want = ref.cached(q[0], k[0], v[0].nan_to_num(), n, **{**dict(K=4, calib="fwm", tau=8.0), **op})
    ref.within(o[0, ..., 32:], want[0][..., 32:], want[1][..., 32:], "other channels")


def test_the_last_positions_of_the_longest_table():
    """A sequence of nearly 2^31 keys whose table names one page, its last: with every
    key in sight, few, one, or more first tokens than positions."""
    d, page, width = 32, 16, (1 << 27) - 1
    cache, _, k, v = filled((12,), 1, d, page, torch.float32, 110)
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, -1] = int((cache.data != 0).flatten(1).any(1).nonzero()[0])
    n = width * page - 4  # the page's 12th token is the newest key
    q = draw((1, 2, 1, d), torch.float32, 114)
    for win, sinks, see in ((1, 0, 1), (5, 0, 5), (1, (1 << 31) - 1, 12), (0, 0, 12)):
        got = kia.cache4_attention(q, cache, table, ints(n), recon="softmax", window=win, sinks=sinks)
        want = ref.cached(q[0], k[0, :, 12 - see:], v[0, :, 12 - see:], see, recon="softmax")
        ref.within(got[0], *want, f"window {win}, {sinks} first tokens")


def test_rows_four_million_elements_apart():
    """Views of one buffer of 9 GB: rows as far apart as the kernels take them, so that
    offsets pass 2^32, forward, backward, rotated, and into the cache."""
    T, d, st = 1040, 32, 1 << 22
    base = torch.empty((T - 1) * st + 4096, dtype=torch.bfloat16, device="cuda")

    def far(x, at):
        y = base.as_strided((1, x.shape[1], T, d), (base.numel(), d, st, 1), at)
        return y.copy_(x)

    q, g = draw((1, 4, T, d), torch.bfloat16, 120), draw((1, 4, T, d), torch.bfloat16, 121)
    k, v = draw((1, 2, T, d), torch.bfloat16, 122), draw((1, 2, T, d), torch.bfloat16, 123)
    x = far(q, 0), far(k, 4 * d), far(v, 6 * d), far(g, 8 * d)
    o, lse = kia.window_forward(q, k, v, 300, 2)
    grads = kia.window_backward(q, k, v, o, g, lse, 300, 2)
    o2, lse2 = far(o, 12 * d).zero_(), torch.empty_like(lse)
    kia.kia_window_fwd(*x[:3], o2, lse2, 300, 2)
    assert torch.equal(o2, o) and torch.equal(lse2, lse)
    to = [far(torch.zeros_like(t), at * d) for t, at in zip(grads, (16, 20, 22))]
    ws = torch.empty(kia.kia_window_ws_bytes(1, 4, 2, T, d, 300, 2), dtype=torch.uint8, device="cuda")
    kia.kia_window_bwd(*x[:3], o2, x[3], lse2, ws, *to, 300, 2)
    assert all(torch.equal(a, b) for a, b in zip(to, grads))
    plan = kia.rotary_plan(d)
    for a, b in zip(kia.rotary(*x[:2], plan, 5), kia.rotary(q, k, plan, 5)):
        assert torch.equal(a, b)
    caches = []
    for keys, values in ((k, v), (x[1], x[2])):
        caches.append(kia.new_cache4(17, 2, 64, d))
        kia.cache4_write(keys, values, caches[-1], torch.arange(17, dtype=torch.int32, device="cuda")[None], ints(0))
    assert torch.equal(caches[0].data, caches[1].data)


@pytest.mark.parametrize("op", (dict(recon="softmax"), dict(recon="nearest", calib="fwm", K=4, tau=8.0)),
                         ids=lambda o: o["recon"])
def test_cache_of_more_than_four_gigabytes(op):
    """The same tokens on the first and on the last pages of a cache of 5.6 GB, written,
    read and attended to."""
    lengths, page, d, Hkv = (700, 256, 3), 256, 128, 8
    pages = 20000
    cache = kia.new_cache4(pages, Hkv, page, d)
    k, v = draw((3, Hkv, 700, d), torch.bfloat16, 130), draw((3, Hkv, 700, d), torch.bfloat16, 131)
    q = draw((3, 16, 2, d), torch.bfloat16, 132)
    low = torch.arange(9, dtype=torch.int32, device="cuda").view(3, 3)
    out = []
    for table in (low, pages - 1 - low):
        kia.cache4_write(k, v, cache, table, ints(0, 0, 0), ints(*lengths))
        out.append((*kia.cache4_read(cache, table, ints(0, 0, 0), 700, torch.bfloat16),
                    kia.cache4_attention(q, cache, table, ints(*lengths), **op)))
    assert all(torch.equal(a, b) for a, b in zip(*out))
    assert out[1][2].any() and not cache.data[9:-9].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("op", (dict(recon="softmax"), dict(recon="lerp", calib="minmax", K=4),
                                dict(recon="nearest", calib="fwm", K=4, tau=8.0)), ids=lambda o: o["recon"])
@pytest.mark.parametrize("H,Hkv,T", ((1, 1, 1), (4, 2, 1), (6, 2, 1), (2, 2, 4), (4, 2, 2), (5, 1, 1), (17, 1, 1)))
@pytest.mark.parametrize("lengths", ((256, 257, 255), (31, 1100, 0)))
def test_rows_of_a_key_head(dtype, op, H, Hkv, T, lengths):
    """One to seventeen rows a key head, around the four that share their columns and the
    sixteen of a tile, and tables around those that take one part."""
    cache, table, k, v = filled(lengths, Hkv, 32, 32, dtype, 140, 0.7)
    check(draw((3, H, T, 32), dtype, 144), cache, table, k, v, lengths, **op)


@pytest.mark.parametrize("op", (dict(recon="softmax"), dict(recon="lerp", calib="fwm", K=4, tau=8.0)),
                         ids=lambda o: o["recon"])
def test_many_sequences_that_share_pages(op):
    """150 sequences, each a start of the same text on the same pages."""
    B, page, d = 150, 16, 64
    cache, table, k, v = filled((1000,), 2, d, page, torch.bfloat16, 150, 0.7)
    lengths = [int(x) for x in torch.randint(0, 1001, (B,), generator=torch.Generator().manual_seed(3))]
    lengths[:4] = 1000, 0, 1, 16
    q = draw((B, 4, 1, d), torch.bfloat16, 154)
    shared = table.expand(B, -1).contiguous()
    check(q, cache, shared, k.expand(B, -1, -1, -1), v.expand(B, -1, -1, -1), lengths, **op)
    check(q, cache, shared, k.expand(B, -1, -1, -1), v.expand(B, -1, -1, -1), lengths, win=50, sinks=20, **op)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window,sinks", ((1, 200), (1, 199), (7, 1 << 30), (200, 5), (199, 1), ((1 << 31) - 1, 0)))
def test_windows_and_first_tokens_of_the_whole_text(dtype, window, sinks):
    from tests.test_gpu_window import check as window_check, inputs
    q, k, v, g = inputs(2, 2, 1, 200, 32, dtype, seed=160)
    window_check(q, k, v, g, window, sinks)


@pytest.mark.parametrize("dtype", TYPES)
def test_captured_training_step(dtype):
    """Rotation, attention and their gradients by autograd inside one graph, replayed with
    new inputs and eager work between, two graphs alive."""
    T = 130
    shapes = ((2, 4, T, 64), (2, 2, T, 64), (2, 2, T, 64), (2, 4, T, 64))
    static = [draw(s, dtype, 170 + i) for i, s in enumerate(shapes)]
    leaves = [t.requires_grad_() for t in static[:3]]
    plan = kia.rotary_plan(64)
    lengths = ints(T, 70)

    def step():
        o = kia.window_attention(*leaves, 40, 2, lengths=lengths, rotary=plan)
        return (o.detach(), *torch.autograd.grad(o, leaves, static[3]))

    step()  # (its graph is gone before the captures: leaves belong to one at a time)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out))
    for turn in range(4):
        with torch.no_grad():
            for i, (t, s) in enumerate(zip(static, shapes)):
                t.copy_(draw(s, dtype, 180 + 4 * turn + i))
            lengths.copy_(ints(T - turn, 70 + turn))
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = step()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want))
