"""Tokens appended to the 4-bit cache on the device: queries and keys turned on their way,
and the bounds of the pages, against their definitions in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2609_33591_amd as kia  # noqa: E402
from tests import around_reference as ref  # noqa: E402
from tests.serve_reference import bounds_of, draw, ints, table_of  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = (torch.float32, torch.bfloat16)


def turned(x, plan, starts):
    """(value, bound) in 64 bits of x [B, heads, T, d] at positions starts[b] + t."""
    pos = torch.tensor(starts, device="cuda")[:, None] + torch.arange(x.shape[2], device="cuda")
    return ref.rotary(x, plan.freq, plan.layout, plan.factor, pos)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,rot,layout", ((128, 128, "half"), (64, 64, "interleaved"), (32, 32, "half"),
                                          (64, 40, "interleaved"), (64, 42, "half"), (128, 96, "half"),
                                          (128, 2, "half"), (32, 30, "interleaved")))
@pytest.mark.parametrize("page", (16, 64, 256))
def test_append(dtype, d, rot, layout, page):
    """Ragged numbers of tokens at odd places, over pages that hold earlier tokens; what is
    not written stays."""
    B, H, Hkv, T = 5, 4, 3, 70
    starts, counts = [0, 5, page - 1, 2 * page - 3, 3 * page + 7], [70, 0, 1, 37, 70]
    table, pages = table_of([s + T for s in starts], page, 7)
    cache, bounds = kia.new_cache4(pages, Hkv, page, d), None
    plan = kia.rotary_plan(rot, layout=layout, scaling="parts", stretch=4.0, original=64)
    old = draw((B, Hkv, max(starts), d), dtype, 1), draw((B, Hkv, max(starts), d), dtype, 2)
    kia.cache4_write(*old, cache, table, ints(*[0] * B), ints(*starts))
    q, k = draw((B, T, H, d), dtype, 3).transpose(1, 2), draw((B, T, Hkv, d), dtype, 4, 3.0).transpose(1, 2)
    v = draw((B, Hkv, T, d), dtype, 5)
    before = cache.data.clone()
    for bounds in (None, torch.full((pages, Hkv, 2, d), 7.0, dtype=torch.bfloat16, device="cuda")):
        cache.data.copy_(before)
        out = kia.cache4_append(q, k, v, cache, table, ints(*starts), plan, ints(*counts), bounds)
        # queries as rotary turns them, every token
        pos = ints(*starts)[:, None] + torch.arange(T, dtype=torch.int32, device="cuda")
        assert torch.equal(out, kia.rotary(q, None, plan, pos)[0])
        ref.within(out, *turned(q, plan, starts), "q")
        held = ref.held(turned(k, plan, starts)[0]), ref.held(v)
        got = kia.cache4_read(cache, table, ints(*starts), T, torch.float32)
        for b, n in enumerate(counts):
            for x, want in zip(got, held):
                assert torch.equal(x[b, :, :n].double(), want[b, :, :n])
        first = kia.cache4_read(cache, table, ints(*[0] * B), max(starts), torch.float32, ints(*starts))
        for b, s in enumerate(starts):
            for x, want in zip(first, old):
                assert torch.equal(x[b, :, :s].double(), ref.held(want)[b, :, :s])
        used = sum(counts) * 2 * Hkv * (d // 2 + d // 32)
        assert 0 < int((cache.data != before).sum()) <= used
    # bounds of the pages that tokens went to, over everything up to the last one
    want = torch.full_like(bounds, 7.0).double()
    for b, (s, n) in enumerate(zip(starts, counts)):
        every = torch.cat((ref.held(old[0])[b, :, :s], held[0][b, :, :n]), 1)
        for w in range(s // page, (s + n - 1) // page + 1 if n else 0):
            want[table[b, w]] = bounds_of(every, s + n, page, w)
    assert torch.equal(bounds.double(), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,page", ((32, 16), (64, 256), (128, 128), (128, 32)))
def test_prompts_over_pages(dtype, d, page):
    """Prompts over several pages, whole and begun, of one head and of many; a NaN in a key makes
    its group's bounds NaN, in that page alone."""
    B, H, Hkv, T = 2, 9, 5, 600
    starts = [page + 3, 0]
    table, pages = table_of([s + T for s in starts], page, 17)
    cache, plan = kia.new_cache4(pages, Hkv, page, d), kia.rotary_plan(d)
    old = draw((B, Hkv, max(starts), d), dtype, 31)
    kia.cache4_write(old, old, cache, table, ints(0, 0), ints(*starts))
    q, k, v = (draw((B, h, T, d), dtype, 32 + i) for i, h in enumerate((H, Hkv, Hkv)))
    k[1, 2, 333, 7] = math.nan
    bounds = kia.new_bounds4(cache)
    out = kia.cache4_append(q, k, v, cache, table, ints(*starts), plan, bounds=bounds)
    ref.within(out, *turned(q, plan, starts), "q")
    held = ref.held(turned(k, plan, starts)[0])
    got = kia.cache4_read(cache, table, ints(*starts), T, torch.float32)
    assert torch.equal(got[0].double().nan_to_num(9e99), held.nan_to_num(9e99))
    assert torch.equal(got[1].double(), ref.held(v))
    for b, s in enumerate(starts):
        every = torch.cat((ref.held(old)[b, :, :s], held[b]), 1)
        for w in range(s // page, (s + T - 1) // page + 1):
            want = bounds_of(every, s + T, page, w)
            assert torch.equal(bounds[table[b, w]].double().nan_to_num(9e99), want.nan_to_num(9e99))
    # the same from what the cache holds
    again = kia.new_bounds4(cache)
    kia.cache4_bounds(cache, again, table, ints(*starts), ints(*(s + T for s in starts)))
    assert torch.equal(again.float().nan_to_num(9e9), bounds.float().nan_to_num(9e9))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ("half", "interleaved"))
def test_keys_at_borders(dtype, layout):
    """A key at position 0 is held as it is: every midpoint and level on either side, least
    and largest magnitudes, where 32 bits cannot decide; infinities and NaNs."""
    one = torch.tensor([0.0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, -0.25,
                        -0.75, -1.25, -1.75, -2.5, -3.5, -5, -6, 0.26, 0.24, 0.74, 0.76, 1.24, 2.52,
                        -3.48, 4.96, -5.04])
    top = torch.finfo(dtype).max
    rows = [one * 2.0 ** e for e in (0, -7, 9, 100, -100)]
    rows += [one.clamp(-s, s) for s in (1.4, 1.5, 1.6, 2.9, 3.0, 3.1, 0.3)]
    rows += [torch.zeros(32), torch.full((32,), top), one / 6 * top]
    bad = [one.clone() for _ in range(3)]
    bad[0][3], bad[1][31], bad[2][0] = math.nan, math.inf, -math.inf
    x = torch.stack(rows).to(dtype).cuda()
    n = len(rows)
    x = torch.cat((torch.cat((x, x.flip(0)), 1), torch.stack([torch.cat((b, one)) for b in bad]).to(dtype).cuda()))
    x = x[:, None, None]  # every row a sequence of one token, two groups of 32
    B = x.shape[0]
    cache = kia.new_cache4(B, 1, 16, 64)
    bounds = kia.new_bounds4(cache)
    table, plan = torch.arange(B, dtype=torch.int32, device="cuda")[:, None], kia.rotary_plan(64, layout=layout)
    q = kia.cache4_append(x, x, x, cache, table, ints(*[0] * B), plan, bounds=bounds)
    assert torch.equal(q[:n], x[:n])
    k, v = kia.cache4_read(cache, table, ints(*[0] * B), 1, torch.float32)
    want = ref.held(x)
    assert torch.equal(k[:n].double(), want[:n])
    assert torch.equal(v.double().nan_to_num(9e99), want.nan_to_num(9e99))
    # a partner's infinity or NaN reaches its pair (0 times it is NaN)
    pair = torch.isnan(turned(x, plan, [0] * B)[0].unflatten(-1, (2, 32))).any(-1)
    inf = ~torch.isfinite(x).unflatten(-1, (2, 32)).all(-1)
    for b in range(n, B):
        nan = torch.isnan(k[b].unflatten(-1, (2, 32))).all(-1)
        assert torch.equal(nan, (pair | inf)[b])
    low = bounds[:n].double()
    assert torch.equal(low[:, 0, 0], want[:n, 0, 0]) and torch.equal(low[:, 0, 1], want[:n, 0, 0])
    nan = torch.isnan(k[n:, 0, 0])
    assert torch.equal(torch.isnan(bounds[n:, 0, 0]), nan) and torch.equal(torch.isnan(bounds[n:, 0, 1]), nan)


@pytest.mark.parametrize("dtype", TYPES)
def test_many_keys_are_rounded_once(dtype):
    """2.6 million turned keys, far positions: each the rounding of the exact rotation."""
    B, Hkv, T, d, page = 4, 5, 1024, 128, 128
    starts = [0, 1000, 99_999, 31_000]
    table = torch.full((B, 800), -1, dtype=torch.int32)
    place = iter(range(100))
    for b, s in enumerate(starts):
        for w in range(s // page, (s + T - 1) // page + 1):
            table[b, w] = next(place)
    cache, plan = kia.new_cache4(100, Hkv, page, d), kia.rotary_plan(d)
    k = draw((B, Hkv, T, d), dtype, 11, 2.0)
    kia.cache4_append(k, k, k, cache, table.cuda(), ints(*starts), plan)
    got = kia.cache4_read(cache, table.cuda(), ints(*starts), T, torch.float32)
    assert torch.equal(got[0].double(), ref.held(turned(k, plan, starts)[0]))
    assert torch.equal(got[1].double(), ref.held(k))


@pytest.mark.parametrize("page", (16, 32, 128))
def test_places_that_are_none(page):
    """Tokens before the first position, past the table and on pages that the cache does not
    have are dropped, their queries turned all the same."""
    d, T = 64, 50
    cache = kia.new_cache4(3, 2, page, d)
    bounds = kia.new_bounds4(cache)
    q, k, v = (draw((3, 2, T, d), torch.float32, i) for i in (1, 2, 3))
    table = torch.tensor([[0, 3], [-1, 1], [2, -2147483648]], dtype=torch.int32, device="cuda")
    starts, plan = [-5, page - 13, 2147483600], kia.rotary_plan(d)
    out = kia.cache4_append(q, k, v, cache, table, ints(*starts), plan, bounds=bounds)
    want, bound = turned(q, plan, starts)
    ref.within(out, want, bound, "q")
    hk = ref.held(turned(k, plan, starts)[0])
    got = kia.cache4_read(cache, table, ints(*starts), T, torch.float32)
    pos = ints(*starts).long()[:, None] + torch.arange(T, device="cuda")
    ok = torch.zeros(3, T, dtype=torch.bool, device="cuda")
    ok[0] = (pos[0] >= 0) & (pos[0] < page)
    ok[1] = (pos[1] >= page) & (pos[1] < 2 * page)
    for x, y in zip(got, (hk, ref.held(v))):
        assert torch.equal(x.double(), torch.where(ok[:, None, :, None], y, 0.0))
    assert not cache.data[2].any() and not bounds[2].any()
    for b, place in ((0, 0), (1, 1)):
        y = hk[b][:, ok[b]]
        assert torch.equal(bounds[place].double(), torch.stack((y.amin(1), y.amax(1)), 1))


@pytest.mark.parametrize("d", (32, 64, 128))
@pytest.mark.parametrize("page", (16, 32, 64, 128, 256))
def test_bounds(d, page):
    """Bounds of written tokens, of a part of the pages, and of a NaN; the others stay."""
    lengths = [3 * page + 5, 1, 0, page, 2 * page - 1]
    table, pages = table_of(lengths, page, 3, width=5)
    cache = kia.new_cache4(pages, 2, page, d)
    k = draw((5, 2, max(lengths), d), torch.bfloat16, 4)
    k[4, 1, page + 2, 5] = math.nan
    n = ints(*lengths)
    kia.cache4_write(k, k, cache, table, torch.zeros_like(n), n)
    bounds = torch.full((pages, 2, 2, d), 5.0, dtype=torch.bfloat16, device="cuda")
    starts, ends = [page + 3, 0, 0, -9, page], [1 << 30, 1, 0, page, 2 * page - 1]
    kia.cache4_bounds(cache, bounds, table, ints(*starts), ints(*ends))
    held, want = ref.held(k), torch.full_like(bounds, 5.0).double()
    for b, (s, e) in enumerate(zip(starts, ends)):
        for w in range(max(s, 0) // page, 5):
            if w * page < min(e, lengths[b]):
                # (past the end the pages hold zeros)
                every = torch.cat((held[b, :, :lengths[b]], torch.zeros(2, page, d, dtype=torch.float64, device="cuda")), 1)
                want[table[b, w]] = bounds_of(every, e, page, w)
    assert torch.equal(torch.isnan(bounds), torch.isnan(want))
    assert torch.equal(bounds.double().nan_to_num(9e99), want.nan_to_num(9e99))
    assert bool(torch.isnan(want).any())


def test_streams_and_capture():
    """On a side stream, and captured: two graphs of a step, replayed with positions that
    move; every replay as the eager call."""
    B, H, Hkv, d, page = 3, 4, 2, 128, 32
    table, pages = table_of([200] * B, page, 1)
    plan = kia.rotary_plan(d)
    q, k, v = (draw((B, h, 2, d), torch.bfloat16, i) for i, h in ((1, H), (2, Hkv), (3, Hkv)))
    caches = [kia.new_cache4(pages, Hkv, page, d) for _ in range(4)]
    bounds = [kia.new_bounds4(c) for c in caches]
    starts = ints(0, 30, 95)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = kia.cache4_append(q, k, v, caches[0], table, starts, plan, bounds=bounds[0])
    torch.cuda.current_stream().wait_stream(side)
    b = kia.cache4_append(q, k, v, caches[1], table, starts, plan, bounds=bounds[1])
    assert torch.equal(a, b) and torch.equal(caches[0].data, caches[1].data) and torch.equal(bounds[0], bounds[1])
    graphs = []
    for i in (2, 3):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = kia.cache4_append(q, k, v, caches[i], table, starts, plan, bounds=bounds[i])
        graphs.append((graph, out))
    caches[1].data.zero_(), bounds[1].zero_()
    for turn in range(4):
        starts.add_(7 * turn)
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = kia.cache4_append(q, k, v, caches[1], table, starts, plan, bounds=bounds[1])
        for i, (_, out) in zip((2, 3), graphs):
            assert torch.equal(out, want)
            assert torch.equal(caches[i].data, caches[1].data) and torch.equal(bounds[i], bounds[1])
