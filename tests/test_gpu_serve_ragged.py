"""Attention behind shared tokens where the texts' remainders differ much: parts by length."""
import pytest

torch = pytest.importorskip("torch")

import paper_2609_33591_amd as kia  # noqa: E402
from tests import around_reference as ref  # noqa: E402
from tests.serve_reference import draw, filled, ints, table_of  # noqa: E402

pytestmark = pytest.mark.gpu
OPS = [dict(recon="softmax"), dict(recon="lerp", calib="minmax", K=4, tau=8.0),
       dict(recon="nearest", calib="fwm", K=16, tau=6.0), dict(recon="lerp", calib="resolved", K=3, tau=8.0)]


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("op", OPS, ids=lambda op: "-".join(str(x) for x in op.values()))
@pytest.mark.parametrize("H,Hkv,T,d,page,shared,lengths", [
    (4, 2, 1, 64, 32, 64, (9000, 65, 64, 63, 0, 2, 70)), (6, 1, 5, 32, 16, 32, (40, 37, 5000, 6, 0, 3000)),
    (16, 1, 1, 128, 256, 512, (513, 512, 4000))])
def test_shared_and_long_remainders(dtype, op, H, Hkv, T, d, page, shared, lengths):
    """One or two long texts among short ones, that end within the shared tokens or at their
    end, rows of one tile and of two; and the same in a table of room for much longer ones."""
    cache, table, _, k, v = filled(lengths, Hkv, d, page, dtype, 180, 0.7, shared)
    q, n = draw((len(lengths), H, T, d), dtype, 184), ints(*lengths)
    o = kia.cache4_attention(q, cache, table, n, shared=shared, **op)
    for b, m in enumerate(lengths):
        want = ref.cached(q[b], k[b, :, :m], v[b, :, :m], m, **{**dict(K=4, calib="fwm", tau=8.0), **op})
        ref.within(o[b], *want, f"sequence {b}")
    wide = torch.cat((table, torch.full((len(lengths), 40000 // page), -1, dtype=torch.int32, device="cuda")), 1)
    y = kia.cache4_attention(q, cache, wide, n, shared=shared, **op)
    for b, m in enumerate(lengths):
        want = ref.cached(q[b], k[b, :, :m], v[b, :, :m], m, **{**dict(K=4, calib="fwm", tau=8.0), **op})
        ref.within(y[b], *want, f"sequence {b}, wide")


@pytest.mark.parametrize("op", OPS[:2], ids=lambda op: op["recon"])
@pytest.mark.parametrize("B,H", ((150, 2), (150, 16), (300, 2)))
def test_shared_and_many_sequences(op, B, H):
    """More sequences than the lanes that count their parts, half of them without a remainder, rows
    that are joined by a workgroup each and by a few lanes; bitwise repeatable, and captured while
    lengths move."""
    d, page, shared = 32, 16, 32
    lengths = [shared + (0 if b % 2 else b) for b in range(B)]
    lengths[77], lengths[131], lengths[B - 1] = 6300, 3000, 4500
    cache, table, _, k, v = filled(tuple(lengths), 1, d, page, torch.bfloat16, 190, 0.7, shared)
    q, n = draw((B, H, 1, d), torch.bfloat16, 194), ints(*lengths)

    def call():
        return kia.cache4_attention(q, cache, table, n, shared=shared, **op)

    o = call()
    for b, m in enumerate(lengths):
        want = ref.cached(q[b], k[b, :, :m], v[b, :, :m], m, **{**dict(K=4, calib="fwm", tau=8.0), **op})
        ref.within(o[b], *want, f"sequence {b}")
    assert torch.equal(call(), o)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = call()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, o)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = call()
    first = n.clone()
    for turn in range(4):
        n.copy_(first.roll(11 * turn))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, call())


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("op", OPS, ids=lambda op: "-".join(str(x) for x in op.values()))
@pytest.mark.parametrize("B,H,Hkv,T,d", ((64, 12, 2, 3, 32), (65, 12, 2, 3, 32), (90, 20, 1, 5, 64)))
def test_long_remainders_of_many_row_tiles(dtype, op, B, H, Hkv, T, d):
    """Sequences of several row tiles, as many as find their parts in each workgroup and more, queries
    before the text and texts that end within the shared tokens among them."""
    page, shared = 32, 64
    lengths = [(shared + b, shared, 1 + b % 70, 0)[b % 4] for b in range(B)]
    lengths[0], lengths[B - 1] = 4700, 5300
    cache, table, _, k, v = filled(tuple(lengths), Hkv, d, page, dtype, 200, 0.7, shared)
    q = draw((B, H, T, d), dtype, 204)
    o = kia.cache4_attention(q, cache, table, ints(*lengths), shared=shared, **op)
    for b, m in enumerate(lengths):
        want = ref.cached(q[b], k[b, :, :m], v[b, :, :m], m, **{**dict(K=4, calib="fwm", tau=8.0), **op})
        ref.within(o[b], *want, f"sequence {b}")


def shortest(call, runs=20):
    times = []
    for _ in range(runs):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b))
    return min(times)


@pytest.mark.parametrize("recon", ("softmax", "lerp"))
def test_one_long_text_is_no_loss(recon):
    """One text of 100 000 tokens of its own among 256: with its remainder in one part the call took
    three times the time that it takes without shared tokens; in parts by length a third."""
    B, H, Hkv, d, page, shared = 256, 16, 4, 128, 64, 8192
    lengths = [shared + 200] * B
    lengths[5] = shared + 100_000
    table, pages = table_of(lengths, page, 3, shared)
    cache = kia.new_cache4(pages, Hkv, page, d)
    cache.data.random_(0, 120)
    q, n, op = draw((B, H, 1, d), torch.bfloat16, 4), ints(*lengths), dict(recon=recon, calib="fwm", K=4, tau=8.0)
    with_shared = shortest(lambda: kia.cache4_attention(q, cache, table, n, shared=shared, **op))
    without = shortest(lambda: kia.cache4_attention(q, cache, table, n, **op))
    assert with_shared < 1.5 * without, (with_shared, without)
