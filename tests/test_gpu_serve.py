"""Selected pages, attention over them, and attention behind shared tokens on the device,
against their definitions in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2609_33591_amd as kia  # noqa: E402
from tests import around_reference as ref  # noqa: E402
from tests.serve_reference import draw, filled, ints, over_pages, select, table_of  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = (torch.float32, torch.bfloat16)
OPS = [dict(recon="softmax")] + [dict(recon=r, calib=c, K=K, tau=t) for r, c, K, t in (
    ("lerp", "minmax", 4, 8.0), ("lerp", "fwm", 16, 6.0), ("lerp", "resolved", 3, 8.0),
    ("nearest", "fwm", 4, 8.0), ("nearest", "minmax", 64, 8.0), ("nearest", "resolved", 2, 6.0))]
FULL = dict(K=4, calib="fwm", tau=8.0)


def name(op):
    return "-".join(str(x) for x in op.values())


def by_table(bounds, table):
    """Bounds [W, Hkv, 2, d] of a sequence's table entries (those of no page: anything)."""
    return bounds[table.long().clamp(0, bounds.shape[0] - 1)]


# ---- selection ----------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hkv,T,d,page,count,first,last", [
    (4, 2, 1, 64, 16, 5, 1, 1), (3, 3, 2, 32, 32, 3, 0, 1), (16, 1, 1, 128, 16, 7, 2, 3),
    (10, 1, 5, 128, 16, 40, 1, 2), (2, 2, 3, 32, 16, 4, 1, 3), (40, 1, 4, 128, 64, 2, 0, 2)])
def test_select(dtype, H, Hkv, T, d, page, count, first, last):
    lengths = (1, 0, 2 * page + 1, 700, 699, 16 * page)
    cache, table, bounds, _, _ = filled(lengths, Hkv, d, page, dtype, 20, 0.7)
    q = draw((len(lengths), H, T, d), dtype, 24)
    got = kia.cache4_select(q, cache, bounds, table, ints(*lengths), count, first, last)
    assert got.shape == (len(lengths), Hkv, T, count) and got.dtype == torch.int32
    for b, n in enumerate(lengths):
        want = select(q[b], by_table(bounds, table[b]), table[b].tolist(), n, page, cache.pages, count, first, last)
        assert got[b].tolist() == want, b


def test_select_far_and_many():
    """More pages than stay in registers; scores that agree in all but low bits; ties."""
    page, n, d = 16, 16 * 5000 + 3, 32
    table = torch.randperm(5001, generator=torch.Generator().manual_seed(2)).int()[None].cuda()
    cache = kia.Cache4(torch.zeros(5001, 2, 1, page * (d // 2 + d // 32), dtype=torch.uint8, device="cuda"), d)
    q = draw((1, 1, 1, d), torch.float32, 3)
    q[0, 0, 0, :2] = torch.tensor([1.0, 2.0 ** -20])
    bounds = draw((5001, 1, 2, d), torch.bfloat16, 4)
    near = torch.ones(5001, 1, 2, d, dtype=torch.bfloat16, device="cuda")
    near[:, 0, :, 1] = torch.randint(1, 100, (5001, 1), generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    same = torch.ones_like(near)
    for x in (bounds, near, same):
        x = torch.stack((x.amin(2), x.amax(2)), 2)
        for count, first, last in ((64, 1, 1), (1000, 0, 7), (4999, 1, 1), (5000, 1, 1), (5001, 3, 3), (9, 4, 5)):
            got = kia.cache4_select(q, cache, x, table, ints(n), count, first, last)
            want = select(q[0], by_table(x, table[0]), table[0].tolist(), n, page, 5001, count, first, last)
            assert got[0].tolist() == want, (count, first, last)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("W", (1024, 1025, 4096, 4097))
def test_select_of_the_most_heads(dtype, W):
    """As many channels a key head as there may be, and tables to either side of what a
    workgroup holds."""
    page, d, H, n = 16, 128, 64, 16 * W - 5
    table = torch.randperm(W, generator=torch.Generator().manual_seed(6)).int()[None].cuda()
    cache = kia.Cache4(torch.zeros(W, 2, 1, page * (d // 2 + d // 32), dtype=torch.uint8, device="cuda"), d)
    q, bounds = draw((1, H, 2, d), dtype, 7), draw((W, 1, 2, d), torch.bfloat16, 8)
    bounds = torch.stack((bounds.amin(2), bounds.amax(2)), 2)
    for count, first, last in ((64, 1, 2), (W - 3, 0, 1)):
        got = kia.cache4_select(q, cache, bounds, table, ints(n), count, first, last)
        want = select(q[0], by_table(bounds, table[0]), table[0].tolist(), n, page, W, count, first, last)
        assert got[0].tolist() == want, (count, first, last)


def test_select_what_is_not_finite():
    """A bound or query of NaN ranks as infinite, whatever else a page has; entries that name
    no page are not taken, first and last ones neither."""
    page, d, lengths = 16, 64, (16 * 12, 16 * 12 - 5)
    cache, table, bounds, _, _ = filled(lengths, 2, d, page, torch.float32, 30)
    q = draw((2, 4, 2, d), torch.float32, 31)
    bounds[table[0, 5].long(), 1, :, 9] = math.nan
    q[1, 0, 1, 3] = math.nan
    q[1, 2, 0, 3] = math.inf
    table[0, 0], table[0, 7], table[1, 11], table[1, 3] = -1, 99999, -5, cache.pages
    got = kia.cache4_select(q, cache, bounds, table, ints(*lengths), 4, 1, 1)
    for b, n in enumerate(lengths):
        want = select(q[b], by_table(bounds, table[b]), table[b].tolist(), n, page, cache.pages, 4, 1, 1)
        assert got[b].tolist() == want
    assert 5 in got[0, 1, 0].tolist() and 0 not in got[0].flatten().tolist()
    # a length past the table is the table's
    got = kia.cache4_select(q, cache, bounds, table[:, :5].contiguous(), ints(1 << 30, 3000), 3)
    for b in range(2):
        want = select(q[b], by_table(bounds, table[b, :5]), table[b, :5].tolist(), 5 * page, page, cache.pages, 3, 1, 1)
        assert got[b].tolist() == want


# ---- over selected pages ---------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("op", OPS, ids=name)
@pytest.mark.parametrize("H,Hkv,T,d,page,count,lengths", [
    (4, 2, 1, 64, 16, 5, (1, 0, 65, 200)), (3, 3, 2, 32, 32, 2, (2, 1, 64, 129)),
    (20, 1, 2, 128, 64, 7, (63, 64, 700)), (10, 1, 5, 128, 16, 33, (5, 3, 700))])
def test_attention_over_selected(dtype, op, H, Hkv, T, d, page, count, lengths):
    cache, table, bounds, k, v = filled(lengths, Hkv, d, page, dtype, 40, 0.7)
    q, n = draw((len(lengths), H, T, d), dtype, 44), ints(*lengths)
    pages = kia.cache4_select(q, cache, bounds, table, n, count)
    o = kia.cache4_attention(q, cache, table, n, pages=pages, **op)
    for b, m in enumerate(lengths):
        want = over_pages(q[b], k[b, :, :m], v[b, :, :m], m, page, pages[b].tolist(), **{**FULL, **op})
        ref.within(o[b], *want, f"sequence {b} {op}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("op", (OPS[0], OPS[1], OPS[4]), ids=name)
def test_lists_of_any_kind(dtype, op):
    """Pages in any order, none in between, numbers past the table or the row's position, a
    page twice, nothing at all."""
    page, d, n = 16, 64, 16 * 9 + 3
    cache, table, _, k, v = filled((n,), 2, d, page, dtype, 50, 0.7)
    q = draw((1, 4, 3, d), dtype, 54)
    lists = torch.tensor([[[9, 0, 3, -1, 5, 2], [-1, -1, -1, -1, -1, -1], [8, 1 << 30, -7, 10, 99, 1]],
                          [[4, 4, 4, 2, 2, 9], [-1, 7, -1, -1, -1, -1], [9, 8, 7, 6, 5, 4]]],
                         dtype=torch.int32, device="cuda")[None]
    o = kia.cache4_attention(q, cache, table, ints(n), pages=lists, **op)
    known = [[[w if w < 10 else -1 for w in x] for x in h] for h in lists[0].tolist()]
    ref.within(o[0], *over_pages(q[0], k[0], v[0], n, page, known, **{**FULL, **op}), "lists")
    assert not o[0, :2, 1].any()
    # entries of the table that name no page
    table[0, 9], table[0, 4] = -1, cache.pages
    o = kia.cache4_attention(q, cache, table, ints(n), pages=lists, **op)
    known = [[[w if w not in (9, 4) else -1 for w in x] for x in h] for h in known]
    ref.within(o[0], *over_pages(q[0], k[0], v[0], n, page, known, **{**FULL, **op}), "no pages")


@pytest.mark.parametrize("op", (OPS[0], OPS[2]), ids=name)
@pytest.mark.parametrize("page,count", ((16, 2500), (256, 150)))
def test_long_lists(op, page, count):
    """Lists of more pages than a part takes, and of more keys than a tile's rows."""
    n, d = page * count, 32
    cache, table, _, k, v = filled((n + 5,), 1, d, page, torch.bfloat16, 60, 0.7)
    q = draw((1, 2, 1, d), torch.bfloat16, 64)
    lists = torch.randperm(count, generator=torch.Generator().manual_seed(6)).int().cuda()[None, None, None]
    o = kia.cache4_attention(q, cache, table, ints(n + 5), pages=lists, **op)
    ref.within(o[0], *ref.cached(q[0], k[0, :, :n], v[0, :, :n], n, **{**FULL, **op}), "long")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("recon", ("lerp", "nearest"))
@pytest.mark.parametrize("alike", (False, True))
def test_window_weights_need_no_more_pages(dtype, recon, alike):
    """A key below the row's maximum by tau weighs nothing under FWM: attention over the pages
    that the bounds let into the window is attention over all. (Of random keys these are all
    pages; of pages whose keys are alike a few.)"""
    page, d, n, tau = 16, 64, 900, 3.0

    def change(k, v):
        if alike:
            mean = draw((57, 1, d), torch.float32, 75, 1.5) + draw((57, page, d), torch.float32, 76, 0.05)
            k[0, 0] = mean.flatten(0, 1)[:n].to(k.device, k.dtype)

    cache, table, bounds, k, v = filled((n,), 1, d, page, dtype, 70, 1.5, change=change)
    q = draw((1, 1, 1, d), dtype, 74, 2.0)
    s = (q[0].double() @ k[0].double().transpose(-1, -2))[0, 0, :n] / math.sqrt(d)
    w = by_table(bounds, table[0]).double()[:, 0]
    top = torch.maximum(q[0, 0, 0].double() * w[:, 0], q[0, 0, 0].double() * w[:, 1]).sum(-1) / math.sqrt(d)
    assert bool((s <= top.repeat_interleave(page)[:n] + 1e-9).all())
    need = int((top >= s.max() - tau).sum()) + 2
    assert not alike or need < 30
    pages = kia.cache4_select(q, cache, bounds, table, ints(n), need)
    op = dict(recon=recon, calib="fwm", K=8, tau=tau)
    want, bound = ref.cached(q[0], k[0], v[0], n, **op)
    ref.within(kia.cache4_attention(q, cache, table, ints(n), pages=pages, **op)[0], want, bound, "selected")
    ref.within(kia.cache4_attention(q, cache, table, ints(n), **op)[0], want, bound, "all")


# ---- behind shared tokens --------------------------------------------------------------
def check_shared(q, cache, table, k, v, lengths, shared, **op):
    o = kia.cache4_attention(q, cache, table, ints(*lengths), shared=shared, **op)
    for b, n in enumerate(lengths):
        want = ref.cached(q[b], k[b, :, :n], v[b, :, :n], n, **{**FULL, **op})
        ref.within(o[b], *want, f"sequence {b} {op}")
    return o


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("op", OPS, ids=name)
@pytest.mark.parametrize("H,Hkv,T,d,page,shared,lengths", [
    (4, 2, 1, 64, 16, 64, (65, 64, 200, 64)), (3, 3, 2, 32, 32, 32, (40, 33, 129)),
    (16, 2, 1, 128, 64, 256, (257, 300, 700, 256, 260)), (10, 1, 5, 128, 256, 512, (515, 700))])
def test_shared(dtype, op, H, Hkv, T, d, page, shared, lengths):
    cache, table, _, k, v = filled(lengths, Hkv, d, page, dtype, 80, 0.7, shared)
    check_shared(draw((len(lengths), H, T, d), dtype, 84), cache, table, k, v, lengths, shared, **op)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("op", (OPS[0], OPS[1], OPS[4]), ids=name)
def test_shared_short_texts(dtype, op):
    """Texts that end within the shared tokens, of length 0, and queries before the text."""
    shared, lengths = 128, (200, 100, 0, 2, 128, 129, 17)
    cache, table, _, k, v = filled((200,) * 7, 2, 64, 16, dtype, 90, 0.7, shared)
    check_shared(draw((7, 6, 4, 64), dtype, 94), cache, table, k, v, lengths, shared, **op)


@pytest.mark.parametrize("op", (OPS[0], OPS[2]), ids=name)
@pytest.mark.parametrize("dtype", TYPES)
def test_shared_many_rows(op, dtype):
    """Row tiles across sequences, keys over many workgroups, an odd number of tiles."""
    B, shared = 37, 2048
    lengths = tuple(shared + (7 * b) % 90 for b in range(B))
    cache, table, _, k, v = filled(lengths, 1, 128, 64, dtype, 100, 0.7, shared)
    check_shared(draw((B, 3, 3, 128), dtype, 104), cache, table, k, v, lengths, shared, **op)


@pytest.mark.parametrize("op", OPS, ids=name)
@pytest.mark.parametrize("d,page,shared", ((128, 64, 512), (64, 16, 288), (32, 256, 256)))
def test_shared_rows_of_many_tiles(op, d, page, shared):
    """Tiles of rows that no sequence fills, texts that end within the shared tokens, keys and
    values of NaN and entries of no page among them."""
    B = 60
    lengths = tuple((shared + (7 * b) % 90, 5 * b, shared, 0)[0 if b % 4 else b // 4 % 4] for b in range(B))
    cache, table, _, k, v = filled((shared + 90,) * B, 1, d, page, torch.bfloat16, 150, 0.7, shared)
    q = draw((B, 3, 3, d), torch.bfloat16, 154)
    o = check_shared(q, cache, table, k, v, lengths, shared, **op)
    # a NaN key and a NaN value of the shared tokens reach the rows that see them, a NaN value
    # its own channels
    clean = cache.data.clone()
    pos = torch.tensor(lengths, device="cuda")[:, None] - 3 + torch.arange(3, device="cuda")
    for at in (9, shared - 20):
        hit = (pos >= at)[:, None].expand(B, 3, 3)
        for which in (0, 1):
            x = [y.clone() for y in kia.cache4_read(cache, table[:1], ints(at), 1, torch.bfloat16)]
            x[which][0, 0, 0, d - 3] = math.nan
            kia.cache4_write(*x, cache, table[:1], ints(at))
            y = kia.cache4_attention(q, cache, table, ints(*lengths), shared=shared, **op)
            assert torch.equal(y[~hit], o[~hit])
            some = slice(0, d) if which == 0 else slice(d - 32, d)
            assert bool(torch.isnan(y[hit][:, some]).all())
            assert which == 0 or torch.equal(y[hit][:, :d - 32], o[hit][:, :d - 32])
            cache.data.copy_(clean)
    # entries of no page are not seen
    if d == 64:
        bad = table.clone()
        bad[0, 3] = cache.pages
        y = kia.cache4_attention(q, cache, bad, ints(*lengths), shared=shared, **op)
        keep = torch.arange(shared + 90, device="cuda") // page != 3
        for b in (1, 2, 17):
            at = keep[:lengths[b]].nonzero()[:, 0]
            ref.within(y[b], *ref.cached(q[b], k[b][:, at], v[b][:, at], len(at), **{**FULL, **op}), "no page")


def test_shared_is_the_first_rows():
    """Only the first sequence's entries are looked at for the shared tokens, and all of a
    table may be shared."""
    cache, table, _, k, v = filled((160, 190), 2, 64, 32, torch.float32, 110, 0.7, 96)
    q = draw((2, 4, 1, 64), torch.float32, 114)
    o = check_shared(q, cache, table, k, v, (160, 190), 96)
    other = table.clone()
    other[1, :3] = 99999
    assert torch.equal(kia.cache4_attention(q, cache, other, ints(160, 190), shared=96), o)
    other = table[:, :3].contiguous()
    check_shared(q, cache, other, k, v, (96, 90), 96, recon="softmax")
    # and entries of no page are not seen
    table[0, 1] = -1
    o = kia.cache4_attention(q, cache, table, ints(160, 190), shared=96, recon="softmax")
    keep = torch.arange(190, device="cuda") // 32 != 1
    for b, n in enumerate((160, 190)):
        at = keep[:n].nonzero()[:, 0]
        want = ref.cached(q[b], k[b][:, at], v[b][:, at], len(at), recon="softmax")
        ref.within(o[b], *want, "no page")


# ---- both ------------------------------------------------------------------------------
@pytest.mark.parametrize("op", (OPS[0], OPS[2]), ids=name)
def test_many_rows_of_few_parts(op):
    """Rows whose parts are joined many to a workgroup."""
    page, d, n = 16, 32, 1000
    cache, table, bounds, k, v = filled((n,) * 16, 1, d, page, torch.bfloat16, 160, 0.7)
    q = draw((16, 128, 1, d), torch.bfloat16, 164)
    pages = kia.cache4_select(q, cache, bounds, table, ints(*[n] * 16), 60)
    o = kia.cache4_attention(q, cache, table, ints(*[n] * 16), pages=pages, **op)
    for b in range(16):
        want = over_pages(q[b], k[b], v[b], n, page, pages[b].tolist(), **{**FULL, **op})
        ref.within(o[b], *want, f"sequence {b}")
    B, shared = 128, 512
    lengths = tuple(shared + b % 50 for b in range(B))
    cache, table, _, k, v = filled(lengths, 2, d, page, torch.bfloat16, 170, 0.7, shared)
    check_shared(draw((B, 32, 1, d), torch.bfloat16, 174), cache, table, k, v, lengths, shared, **op)


def test_past_four_gigabytes():
    """Pages, bounds and lists at the end of a cache of 4.4 GB."""
    page, d, Hkv, pages = 256, 128, 8, 15_800
    data = torch.empty(pages, 2, Hkv, page * (d // 2 + d // 32), dtype=torch.uint8, device="cuda")
    cache = kia.Cache4(data, d)
    bounds = torch.empty(pages, Hkv, 2, d, dtype=torch.bfloat16, device="cuda")
    table = torch.arange(pages - 1, pages - 9, -1, dtype=torch.int32, device="cuda").view(2, 4)
    table[1, 0] = table[0, 0]  # a shared first page
    n, T = 4 * page - 5, 4 * page - 5
    k, v = draw((2, Hkv, T, d), torch.bfloat16, 1, 0.7), draw((2, Hkv, T, d), torch.bfloat16, 2)
    k[1, :, :page], v[1, :, :page] = k[0, :, :page], v[0, :, :page]
    plan = kia.RotaryPlan(torch.zeros(d // 2, dtype=torch.float64, device="cuda"))  # turns nothing
    x = kia.cache4_append(k[1:], k[1:], v[1:], cache, table[1:].contiguous(), ints(0), plan, bounds=bounds)
    x = kia.cache4_append(k[:1], k[:1], v[:1], cache, table[:1].contiguous(), ints(0), plan, bounds=bounds)
    assert torch.equal(x, k[:1])
    q, lens, hk, hv = draw((2, 16, 1, d), torch.bfloat16, 3), ints(n, n), ref.held(k), ref.held(v)
    got = kia.cache4_select(q, cache, bounds, table, lens, 3)
    o = kia.cache4_attention(q, cache, table, lens, pages=got, recon="softmax")
    y = kia.cache4_attention(q, cache, table, lens, shared=page, recon="softmax")
    for b in range(2):
        want = select(q[b], by_table(bounds, table[b]), table[b].tolist(), n, page, pages, 3, 1, 1)
        assert got[b].tolist() == want
        ref.within(o[b], *over_pages(q[b], hk[b], hv[b], n, page, want, recon="softmax"), "pages")
        ref.within(y[b], *ref.cached(q[b], hk[b], hv[b], n, recon="softmax"), "shared")


def calls(cache, table, bounds, n, T, H, d, dtype, seed, op, shared):
    q = draw((table.shape[0], H, T, d), dtype, seed)
    pages = torch.arange(table.shape[1], dtype=torch.int32, device="cuda").expand(
        table.shape[0], cache.heads, T, -1).contiguous()
    return q, ((lambda c, q: kia.cache4_attention(q, c, table, n, pages=pages, **op)),
               (lambda c, q: kia.cache4_attention(q, c, table, n, shared=shared, **op)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("op", (OPS[0], OPS[1], OPS[4]), ids=name)
@pytest.mark.parametrize("which", (0, 1), ids=("pages", "shared"))
def test_what_is_not_seen_has_no_influence(dtype, op, which):
    """Bytes behind the lengths and pages of others hold anything; keys and values of NaN
    reach the rows that see them and no other; a query of NaN its own row."""
    lengths, T, shared = (150, 77), 4, 64
    cache, table, bounds, k, v = filled(lengths, 1, 64, 16, dtype, 120, 0.7, shared)
    n = ints(*lengths)
    q, both = calls(cache, table, bounds, n, T, 2, 64, dtype, 124, op, shared)
    call = both[which]
    o = call(cache, q)
    for b, m in enumerate(lengths):
        ref.within(o[b], *ref.cached(q[b], k[b, :, :m], v[b, :, :m], m, **{**FULL, **op}), "plain")
    noise = kia.Cache4(torch.randint(0, 256, cache.data.shape, dtype=torch.uint8,
                                     generator=torch.Generator().manual_seed(5)).cuda(), 64)
    noise.data[::3] = 255
    both = [kia.cache4_read(cache, table, ints(0, 0), 150, dtype)[i] for i in (0, 1)]
    kia.cache4_write(*both, noise, table, ints(0, 0), n)
    assert torch.equal(call(noise, q), o)
    # the token at 148 of sequence 0 is seen by its queries 2 and 3, the one at 20 by all
    for at, rows in ((148, [(0, 2), (0, 3)]), (20, [(b, t) for b in (0, 1) for t in range(4)])):
        hit = torch.zeros(2, T, dtype=torch.bool)
        for b, t in rows:
            hit[b, t] = True
        for i in (0, 1):
            x = [y[:, :, at:at + 1].clone() for y in both]
            x[i][0, 0, 0, 40] = math.nan
            kia.cache4_write(*x, noise, table, ints(at, at), ints(1, 0))
            y = call(noise, q).transpose(1, 2)
            z = o.transpose(1, 2)
            assert torch.equal(y[~hit], z[~hit])
            if i == 0:
                assert bool(torch.isnan(y[hit]).all())
            else:
                assert bool(torch.isnan(y[hit][..., 32:]).all()) and torch.equal(y[hit][..., :32], z[hit][..., :32])
            kia.cache4_write(*(y[:, :, at:at + 1] for y in both), noise, table, ints(at, at), ints(1, 0))
    bad = q.clone()
    bad[0, 1, 3, 9] = math.nan
    y = call(cache, bad)
    assert bool(torch.isnan(y[0, 1, 3]).all())
    y[0, 1, 3] = o[0, 1, 3]
    assert torch.equal(y, o)


@pytest.mark.parametrize("op", (OPS[0], OPS[1], OPS[5]), ids=name)
def test_rows_of_equal_scores(op):
    """A query of zeros: every score 0, every weight the same."""
    lengths, shared = (130, 64), 64
    cache, table, bounds, k, v = filled(lengths, 1, 64, 64, torch.float32, 130, 0.7, shared)
    q, both = calls(cache, table, bounds, ints(*lengths), 1, 2, 64, torch.float32, 1, op, shared)
    for call in both:
        o = call(cache, torch.zeros_like(q))
        for b, n in enumerate(lengths):
            bound = (n + 16) * ref.E * v[b, :, :n].abs().mean(1).expand(2, 64) * 4 + 1e-30
            ref.within(o[b, :, 0], v[b, :, :n].mean(1).expand(2, 64), bound, "mean")


@pytest.mark.parametrize("which", (0, 1), ids=("pages", "shared"))
def test_views_streams_and_capture(which):
    """Strided queries, a side stream, and a captured step (append, select, attend) replayed
    while positions move; two graphs with workspaces of their own."""
    page, d, shared, H, Hkv = 32, 128, 128, 8, 2
    lengths = (600, 133, 250)
    cache, table, bounds, k, v = filled(lengths, Hkv, d, page, torch.bfloat16, 140, 0.7, shared, width=20)
    q = draw((3, 2, H, d), torch.bfloat16, 144).transpose(1, 2)
    nk, nv = draw((3, 2, Hkv, d), torch.bfloat16, 145).transpose(1, 2), draw((3, Hkv, 2, d), torch.bfloat16, 146)
    op, plan, n = dict(recon="lerp", calib="fwm", K=4, tau=8.0), kia.rotary_plan(d), ints(*lengths)

    def step(starts, lens):
        x = kia.cache4_append(q, nk, nv, cache, table, starts, plan, bounds=bounds)
        if which:
            return x, kia.cache4_attention(x, cache, table, lens, shared=shared, **op)
        pages = kia.cache4_select(x, cache, bounds, table, lens, 6)
        return pages, kia.cache4_attention(x, cache, table, lens, pages=pages, **op)

    a, o = step(n - 2, n)
    assert torch.equal(o, step(n - 2, n)[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b, y = step(n - 2, n)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, b) and torch.equal(y, o)
    starts, lens = n - 2, n.clone()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(starts, lens)
        graphs.append((graph, out))
    for turn in range(4):
        starts.copy_(n - 2 + turn)
        lens.copy_(n + turn)
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = step(starts, lens)
        for _, out in graphs:
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("op", (OPS[0], OPS[4], dict(recon="lerp", calib="minmax", K=16)), ids=name)
def test_serving(dtype, op):
    """A shared prompt and the texts behind it, token by token: appended with their bounds,
    attended behind the shared tokens and over selected pages."""
    B, H, Hkv, d, page, steps, shared = 3, 6, 2, 64, 16, 5, 64
    prompts = [70, 64, 97]
    plan = kia.rotary_plan(64)
    table, pages = table_of([n + steps for n in prompts], page, 3, shared)
    cache = kia.new_cache4(pages, Hkv, page, d)
    bounds = kia.new_bounds4(cache)
    T = max(prompts) + steps
    q, k, v = draw((B, H, T, d), dtype, 5), draw((B, Hkv, T, d), dtype, 6, 0.7), draw((B, Hkv, T, d), dtype, 7)
    k[:, :, :shared], v[:, :, :shared] = k[:1, :, :shared], v[:1, :, :shared]
    pos = torch.arange(T, device="cuda").expand(B, T)
    hk, hv = ref.held(ref.rotary(k, plan.freq, plan.layout, plan.factor, pos)[0]), ref.held(v)
    lengths = ints(*prompts)
    # the shared tokens by the first sequence, what lies behind by each
    kia.cache4_append(q[:1, :, :shared], k[:1, :, :shared], v[:1, :, :shared], cache, table[:1].contiguous(), ints(0),
                      plan, bounds=bounds)
    rest = [t[:, :, shared:max(prompts)] for t in (q, k, v)]
    kia.cache4_append(*rest, cache, table, ints(*[shared] * B), plan, lengths - shared, bounds)
    for step in range(steps):
        at = lengths.long()[:, None, None, None].expand(B, 1, 1, d)
        tok = [t.gather(2, at.expand(B, t.shape[1], 1, d)) for t in (q, k, v)]
        x = kia.cache4_append(*tok, cache, table, lengths, plan, bounds=bounds)
        lengths += 1
        o = kia.cache4_attention(x, cache, table, lengths, shared=shared, **op)
        pages = kia.cache4_select(x, cache, bounds, table, lengths, 3)
        y = kia.cache4_attention(x, cache, table, lengths, pages=pages, **op)
        for b, m in enumerate(lengths.tolist()):
            ref.within(o[b], *ref.cached(x[b], hk[b, :, :m], hv[b, :, :m], m, **{**FULL, **op}), "shared")
            want = over_pages(x[b], hk[b, :, :m], hv[b, :, :m], m, page, pages[b].tolist(), **{**FULL, **op})
            ref.within(y[b], *want, "selected")
            known = torch.stack([torch.stack((z.amin(1), z.amax(1)), 1) for z in hk[b, :, :m].split(page, 1)])
            assert select(x[b], known, table[b].tolist(), m, page, cache.pages, 3, 1, 1) == pages[b].tolist()
