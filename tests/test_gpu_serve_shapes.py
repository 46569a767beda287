"""Launch shapes of selection and of the attention's join that ordinary batches reach and small
tests do not."""
import pytest

torch = pytest.importorskip("torch")

import paper_2609_33591_amd as kia  # noqa: E402
from tests import around_reference as ref  # noqa: E402
from tests.serve_reference import draw, filled, ints, over_pages, select  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = (torch.float32, torch.bfloat16)
OPS = [dict(recon="softmax"), dict(recon="lerp", calib="fwm", K=16, tau=6.0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("W", (1030, 2049))
@pytest.mark.parametrize("B,Hkv", ((8, 4), (16, 8), (64, 8)))
def test_selections_in_large_batches(dtype, W, B, Hkv):
    """As many selections as let a workgroup rank 128 to 1024 pages (by 256 compute units), texts
    that end to either side of such a batch; fewer candidates than pages asked for, and more."""
    page, d, G, pool = 16, 32, 2, 2100
    g = torch.Generator().manual_seed(6)
    table = torch.stack([torch.randperm(pool, generator=g)[:W] for _ in range(B)]).int().cuda()
    cache = kia.Cache4(torch.zeros(pool, 2, Hkv, page * (d // 2 + d // 32), dtype=torch.uint8, device="cuda"), d)
    x = draw((pool, Hkv, 2, d), torch.bfloat16, 8)
    bounds = torch.stack((x.amin(2), x.amax(2)), 2)
    ends = [1, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1023, 1024, 1025, W - 1, W]
    lengths = [page * ends[(5 * b) % len(ends)] - b % page for b in range(B)]
    q = draw((B, Hkv * G, 1, d), dtype, 7)
    for count, first, last in ((40, 1, 2), (1500, 0, 1)):
        got = kia.cache4_select(q, cache, bounds, table, ints(*lengths), count, first, last)
        for b in range(0, B, 1 + B // 20):
            want = select(q[b], bounds[table[b].long()], table[b].tolist(), lengths[b], page, pool, count, first, last)
            assert got[b].tolist() == want, (b, count)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("op", OPS, ids=lambda op: op["recon"])
@pytest.mark.parametrize("d", (32, 64, 128))
def test_many_rows_of_few_parts(dtype, op, d):
    """Rows whose parts are joined by a few lanes each, of every type and head size, over pages and
    behind shared tokens."""
    full = {**dict(K=4, calib="fwm", tau=8.0), **op}
    page, n, B = 16, 1000, 16
    cache, table, bounds, k, v = filled((n,) * B, 2, d, page, dtype, 160, 0.7)
    q = draw((B, 128, 1, d), dtype, 164)
    pages = kia.cache4_select(q, cache, bounds, table, ints(*[n] * B), 60)
    o = kia.cache4_attention(q, cache, table, ints(*[n] * B), pages=pages, **op)
    for b in range(B):
        ref.within(o[b], *over_pages(q[b], k[b], v[b], n, page, pages[b].tolist(), **full), f"pages, sequence {b}")
    B, shared = 66, 256
    lengths = tuple(shared + b % 50 for b in range(B))
    cache, table, _, k, v = filled(lengths, 2, d, page, dtype, 170, 0.7, shared)
    q = draw((B, 32, 1, d), dtype, 174)
    o = kia.cache4_attention(q, cache, table, ints(*lengths), shared=shared, **op)
    for b, m in enumerate(lengths):
        ref.within(o[b], *ref.cached(q[b], k[b, :, :m], v[b, :, :m], m, **full), f"shared, sequence {b}")
