"""The 4-bit key/value cache and attention over it on the device, against their
definitions in 64 bits (around_reference.held, around_reference.cached)."""
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


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def table_of(lengths, page, seed, spare=2, width=None):
    """Pages in random order, and how many there are."""
    need = [(n + page - 1) // page for n in lengths]
    order = torch.randperm(sum(need) + spare, generator=torch.Generator().manual_seed(seed)).tolist()
    t = torch.full((len(lengths), max(1, width or max(need))), -1, dtype=torch.int32)
    for b, n in enumerate(need):
        for i in range(n):
            t[b, i] = order.pop()
    return t.cuda(), sum(need) + spare


def filled(lengths, Hkv, d, page, dtype, seed, scale=1.0, change=None):
    """A cache of random tokens, its table, and the values it stands for."""
    table, pages = table_of(lengths, page, seed)
    cache = kia.new_cache4(pages, Hkv, page, d)
    T = max(max(lengths), 1)
    k, v = draw((len(lengths), Hkv, T, d), dtype, seed + 1, scale), draw((len(lengths), Hkv, T, d), dtype, seed + 2)
    k[..., ::16] *= 3
    if change:
        change(k, v)
    kia.cache4_write(k, v, cache, table, ints(*[0] * len(lengths)), ints(*lengths))
    return cache, table, ref.held(k), ref.held(v)


# ---- holding tokens ---------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", (32, 64, 128))
@pytest.mark.parametrize("page", (16, 64, 256))
def test_write_and_read(dtype, d, page):
    """Ragged numbers of new tokens at odd places; what is not written stays."""
    B, Hkv, T = 4, 3, 37
    starts, counts = [0, 5, page - 1, 2 * page - 3], [37, 0, 1, 20]
    table, pages = table_of([s + T for s in starts], page, 7)
    cache = kia.new_cache4(pages, Hkv, page, d)
    cache.data.copy_(torch.randint(0, 255, cache.data.shape, dtype=torch.uint8,
                                   generator=torch.Generator().manual_seed(3)))
    before = cache.data.clone()
    old = kia.cache4_read(cache, table, ints(*starts), T, torch.float32)
    k, v = draw((B, T, Hkv, d), dtype, 8).transpose(1, 2), draw((B, Hkv, T, d), dtype, 9, 40.0)
    kia.cache4_write(k, v, cache, table, ints(*starts), ints(*counts))
    got = kia.cache4_read(cache, table, ints(*starts), T, torch.float32)
    for x, y, o in zip(got, (k, v), old):
        want = ref.held(y)
        for b, n in enumerate(counts):
            assert torch.equal(x[b, :, :n].double(), want[b, :, :n])
            assert torch.equal(x[b, :, n:], o[b, :, n:])
    # as many bytes as the tokens have changed, at most
    used = sum(counts) * 2 * Hkv * (d // 2 + d // 32)
    assert 0 < int((cache.data != before).sum()) <= used
    # bfloat16 holds every value
    half = kia.cache4_read(cache, table, ints(*starts), T, torch.bfloat16)
    assert all(torch.equal(a.float(), b) for a, b in zip(half, got))


@pytest.mark.parametrize("dtype", TYPES)
def test_values_at_borders(dtype):
    """Every midpoint and level on either side, groups of zeros, of the least and
    largest magnitudes, and of infinities and NaNs."""
    one = torch.tensor([0.0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, -0.25,
                        -0.75, -1.25, -1.75, -2.5, -3.5, -5, -6, 0.26, 0.24, 0.74, 0.76, 1.24, 2.52,
                        -3.48, 4.96, -5.04])
    top = torch.finfo(dtype).max
    rows = [one * 2.0 ** e for e in (0, -7, 9, 100, -100)]
    rows += [one.clamp(-s, s) for s in (1.4, 1.5, 1.6, 2.9, 3.0, 3.1, 0.3)]
    rows += [torch.zeros(32), torch.full((32,), 2.0 ** -130), torch.full((32,), top), one / 6 * top]
    bad = [one.clone() for _ in range(3)]
    bad[0][3], bad[1][31], bad[2][0] = math.nan, math.inf, -math.inf
    x = torch.stack(rows + bad).to(dtype).cuda()[None, None]
    T = x.shape[2]
    table, pages = table_of([T], 32, 1)
    cache = kia.new_cache4(pages, 1, 32, 32)
    kia.cache4_write(x, x.flip(2), cache, table, ints(0))
    for got, want in zip(kia.cache4_read(cache, table, ints(0), T, torch.float32), (x, x.flip(2))):
        want = ref.held(want)
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got.double().nan_to_num(9e99), want.nan_to_num(9e99))


def test_places_that_are_none():
    """Tokens before the first position, past the table and on pages that the cache
    does not have are dropped, and read as zeros."""
    d, page, T = 64, 16, 50
    cache = kia.new_cache4(3, 2, page, d)
    k, v = draw((3, 2, T, d), torch.float32, 1), draw((3, 2, T, d), torch.float32, 2)
    table = torch.tensor([[0, 3], [-1, 1], [2, -2147483648]], dtype=torch.int32, device="cuda")
    starts = ints(-5, 3, 2147483600)
    kia.cache4_write(k, v, cache, table, starts)
    got = kia.cache4_read(cache, table, starts, T, torch.float32)
    pos = starts.long()[:, None] + torch.arange(T, device="cuda")
    ok = torch.zeros(3, T, dtype=torch.bool, device="cuda")
    ok[0] = (pos[0] >= 0) & (pos[0] < 16)
    ok[1] = (pos[1] >= 16) & (pos[1] < 32)
    for x, y in zip(got, (k, v)):
        assert torch.equal(x.double(), torch.where(ok[:, None, :, None], ref.held(y), 0.0))
    assert not cache.data[2].any()


# ---- attention ----------------------------------------------------------------------
OPS = [dict(recon="softmax")] + [dict(recon=r, calib=c, K=K, tau=t) for r, c, K, t in (
    ("lerp", "minmax", 4, 8.0), ("lerp", "fwm", 16, 6.0), ("lerp", "resolved", 3, 8.0),
    ("nearest", "fwm", 4, 8.0), ("nearest", "minmax", 64, 8.0), ("nearest", "resolved", 2, 6.0),
    ("lerp", "minmax", 1, 8.0))]


def check(q, cache, table, k, v, lengths, win=0, sinks=0, **op):
    o = kia.cache4_attention(q, cache, table, ints(*lengths), window=win, sinks=sinks, **op)
    for b, n in enumerate(lengths):
        want = ref.cached(q[b], k[b, :, :n], v[b, :, :n], n, win=win, sinks=sinks,
                          **{**dict(K=4, calib="fwm", tau=8.0), **op})
        ref.within(o[b], *want, f"sequence {b} {op}")
    return o


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("op", OPS, ids=lambda o: "-".join(str(x) for x in o.values()))
@pytest.mark.parametrize("H,Hkv,T,d,page,lengths", [
    (4, 2, 1, 64, 16, (1, 0, 65, 200)), (3, 3, 2, 32, 32, (2, 1, 64, 129)),
    (16, 2, 1, 128, 64, (63, 64, 300)), (10, 1, 5, 128, 256, (5, 3, 700))])
def test_weights_and_layouts(dtype, op, H, Hkv, T, d, page, lengths):
    cache, table, k, v = filled(lengths, Hkv, d, page, dtype, 20, 0.7)
    check(draw((len(lengths), H, T, d), dtype, 24), cache, table, k, v, lengths, **op)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("op", (OPS[0], OPS[1], OPS[4]), ids=lambda o: "-".join(str(x) for x in o.values()))
@pytest.mark.parametrize("win,sinks", ((1, 0), (1, 1), (63, 5), (64, 64), (130, 70), (5000, 9)))
def test_windows(dtype, op, win, sinks):
    lengths = (700, 65, 3, 511)
    cache, table, k, v = filled(lengths, 2, 64, 16, dtype, 30, 0.7)
    check(draw((4, 6, 3, 64), dtype, 34), cache, table, k, v, lengths, win, sinks, **op)


@pytest.mark.parametrize("op", (OPS[0], OPS[2]), ids=lambda o: o["recon"])
def test_many_rows_and_long_texts(op):
    """More rows than a tile, keys over many workgroups, and a single sequence."""
    cache, table, k, v = filled((4100, 37), 1, 128, 64, torch.bfloat16, 40, 0.7)
    check(draw((2, 24, 7, 128), torch.bfloat16, 44), cache, table, k, v, (4100, 37), **op)
    cache, table, k, v = filled((9001,), 2, 32, 128, torch.float32, 50, 0.7)
    check(draw((1, 2, 1, 32), torch.float32, 54), cache, table, k, v, (9001,), **op)


@pytest.mark.parametrize("op", (OPS[0], OPS[1], OPS[2], OPS[4], OPS[5]), ids=lambda o: "-".join(str(x) for x in o.values()))
def test_rows_of_equal_scores(op):
    """A query of zeros: every score 0, every weight the same."""
    lengths = (130, 1)
    cache, table, k, v = filled(lengths, 1, 64, 64, torch.float32, 60)
    q = torch.zeros(2, 2, 1, 64, device="cuda")
    o = kia.cache4_attention(q, cache, table, ints(*lengths), **op)
    for b, n in enumerate(lengths):
        want = v[b, :, :n].mean(1)
        ref.within(o[b, :, 0], want.expand(2, 64), (n + 16) * ref.E * v[b, :, :n].abs().mean(1).expand(2, 64) * 4 + 1e-30, "mean")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("op", (OPS[0], OPS[1], OPS[4]), ids=lambda o: "-".join(str(x) for x in o.values()))
def test_what_is_not_seen_has_no_influence(dtype, op):
    """Bytes behind the lengths and pages of others hold anything; keys and values of
    NaN reach the rows that see them and no other."""
    lengths, H, T, at = (150, 77), 2, 4, 148
    cache, table, k, v = filled(lengths, 1, 64, 16, dtype, 70, 0.7)
    q = draw((2, H, T, 64), dtype, 74)
    o = check(q, cache, table, k, v, lengths, **op)
    noise = kia.Cache4(torch.randint(0, 256, cache.data.shape, dtype=torch.uint8,
                                     generator=torch.Generator().manual_seed(5)).cuda(), 64)
    noise.data[::3] = 255
    both = [kia.cache4_read(cache, table, ints(0, 0), 160, dtype)[i] for i in (0, 1)]
    kia.cache4_write(*both, noise, table, ints(0, 0), ints(*lengths))
    assert torch.equal(kia.cache4_attention(q, noise, table, ints(*lengths), **op), o)
    # the token at 148 of sequence 0 is seen by queries 2 and 3
    for which in (0, 1):
        x = [t[:, :, at:at + 1].clone() for t in both]
        x[which][0, 0, 0, 40] = math.nan
        kia.cache4_write(*x, noise, table, ints(at, at), ints(1, 0))
        y = kia.cache4_attention(q, noise, table, ints(*lengths), **op)
        assert torch.equal(y[0, :, :2], o[0, :, :2]) and torch.equal(y[1], o[1])
        if which == 0:
            assert bool(torch.isnan(y[0, :, 2:]).all())
        else:
            assert bool(torch.isnan(y[0, :, 2:, 32:]).all())
            assert torch.equal(y[0, :, 2:, :32], o[0, :, 2:, :32])
        kia.cache4_write(*(t[:, :, at:at + 1] for t in both), noise, table, ints(at, at), ints(1, 0))
    # a query of NaN is NaN, and no other
    z = q.clone()
    z[0, 1, 3, 9] = math.nan
    y = kia.cache4_attention(z, cache, table, ints(*lengths), **op)
    assert bool(torch.isnan(y[0, 1, 3]).all())
    y[0, 1, 3] = o[0, 1, 3]
    assert torch.equal(y, o)


def test_pages_that_are_none():
    """Positions on entries that name no page, and past the table, are not seen."""
    d, page = 64, 16
    cache, table, k, v = filled((100,), 1, d, page, torch.float32, 80)
    q = draw((1, 2, 1, d), torch.float32, 84)
    broken = table.clone()
    broken[0, 1], broken[0, 4] = 99999, -7
    keep = torch.ones(100, dtype=torch.bool, device="cuda")
    keep[16:32] = keep[64:80] = False
    o = kia.cache4_attention(q, cache, broken, ints(100), recon="softmax")
    want, bound = ref.cached(q[0], k[0][:, keep], v[0][:, keep], 68, recon="softmax")
    ref.within(o[0], want, bound, "other pages")
    # a length past the table is the table's
    short = table[:, :3].contiguous()
    o = kia.cache4_attention(q, cache, short, ints(100), recon="softmax")
    want, bound = ref.cached(q[0], k[0][:, :48], v[0][:, :48], 48, recon="softmax")
    ref.within(o[0], want, bound, "short table")
    none = torch.full_like(table, -1)
    for recon in ("softmax", "lerp", "nearest"):
        assert not kia.cache4_attention(q, cache, none, ints(100), recon=recon).any()
        assert not kia.cache4_attention(q, cache, table, ints(-4), recon=recon).any()


def test_views_streams_and_capture():
    lengths = (600, 33, 250)
    cache, table, k, v = filled(lengths, 2, 128, 64, torch.bfloat16, 90, 0.7)
    flat = draw((3, 2, 8, 128), torch.bfloat16, 94)
    q = flat.transpose(1, 2)
    op = dict(recon="lerp", calib="fwm", K=4, tau=8.0)
    o = check(q, cache, table, k, v, lengths, **op)
    assert torch.equal(o, kia.cache4_attention(q.contiguous(), cache, table, ints(*lengths), **op))
    n = ints(*lengths)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = kia.cache4_attention(q, cache, table, n, **op)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, o)
    # a captured step: the token's key and value written, attention over them, with
    # lengths that move between replays; two graphs with workspaces of their own
    new = draw((2, 3, 2, 2, 128), torch.bfloat16, 95)
    starts, lens = n.clone() - 2, n.clone()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kia.cache4_write(new[0], new[1], cache, table, starts)
            out = kia.cache4_attention(q, cache, table, lens, **op)
        graphs.append((graph, out))
    for turn in range(4):
        starts.copy_(n - 2 - turn)
        lens.copy_(n - turn)
        for graph, out in graphs:
            graph.replay()
        torch.cuda.synchronize()
        kia.cache4_write(new[0], new[1], cache, table, starts)
        want = kia.cache4_attention(q, cache, table, lens, **op)
        assert all(torch.equal(out, want) for _, out in graphs)
