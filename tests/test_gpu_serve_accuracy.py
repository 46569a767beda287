"""Errors of the operators that serve from the 4-bit cache where single roundings would show:
large scores, small ranks, far angles."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2609_33591_amd as kia  # noqa: E402
from tests import around_reference as ref  # noqa: E402
from tests.serve_reference import draw, ints, select, table_of  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", (32, 64, 128))
@pytest.mark.parametrize("B,G", ((3, 4), (40, 16)))
@pytest.mark.parametrize("score", (100, 700))
def test_shared_weights_of_large_scores(d, B, G, score):
    """Scores near `score` that fp32 holds exactly, one to a wave's keys and one to the sequence's
    own: their weights agree however large the scores. All other keys weigh e^-score."""
    page, shared = 16, 128
    n, at = shared + 5, [5, 40, 70, 101, shared + 2]
    table, pages = table_of((n,) * B, page, 3, shared)
    cache = kia.new_cache4(pages, 1, page, d)
    k, v = torch.zeros(B, 1, n, d, device="cuda"), draw((B, 1, n, d), torch.float32, 5)
    v[:, :, :shared] = v[:1, :, :shared]
    for i, j in enumerate(at):
        k[:, 0, j, i] = 6.0
    kia.cache4_write(k, v, cache, table, ints(*[0] * B))
    q = torch.zeros(B, G, 1, d)
    q[..., :5] = round(score * math.sqrt(d) / 6) + torch.randint(
        0, 128, (B, G, 1, 5), generator=torch.Generator().manual_seed(7)) / 64
    q, v = q.cuda(), ref.held(v)[:, :, at]
    p = torch.softmax(6 * q.double()[..., :5] / math.sqrt(d), -1)
    # In roundings of fp32, weights that are up to 3.1 powers of two apart: the factor of the scores
    # (3) and the differences from maxima (3: weight, waves, parts) times 3.1 ln 2, three
    # exponentials (2 each), products and sums (8): 27, and as many in the sum of the weights,
    # whose reciprocal and product are 3 more
    bound = 60 * ref.E * (p @ v.abs()) + 1e-30
    for m in (0, shared):
        o = kia.cache4_attention(q, cache, table, ints(*[n] * B), recon="softmax", shared=m)
        ref.within(o, p @ v, bound, f"{m} shared")


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("W", (200, 1100))
@pytest.mark.parametrize("scales", ((-40, -40), (-66, -66), (-70, -70), (-72, -72), (-75, -75), (-80, -80), (-20, -125),
                                    (-125, -20), (-100, -120), (62, 62), (100, 24)))
def test_select_of_any_magnitude(dtype, W, scales):
    """Ranks whose fp32 sums would be rounded to few bits, to none, or pass fp32's range: the
    selection is that of the sums in 64 bits, by one workgroup a token and by two launches."""
    page, d, H, count = 16, 64, 4, 50
    table = torch.randperm(W, generator=torch.Generator().manual_seed(6)).int()[None].cuda()
    cache = kia.Cache4(torch.zeros(W, 2, 1, page * (d // 2 + d // 32), dtype=torch.uint8, device="cuda"), d)
    q, x = ((draw(s, torch.float32, i).double() * 2.0 ** e).float()
            for s, i, e in (((1, H, 2, d), 11, scales[0]), ((W, 1, 2, d), 12, scales[1])))
    q, x, n = q.to(dtype), torch.stack((x.amin(2), x.amax(2)), 2).bfloat16(), 16 * W - 3
    got = kia.cache4_select(q, cache, x, table, ints(n), count)
    want = select(q[0], x[table[0].long()], table[0].tolist(), n, page, W, count, 1, 1)
    assert got[0].tolist() == want


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("layout,rot", (("half", 128), ("interleaved", 128), ("half", 72)))
@pytest.mark.parametrize("freq,start", ((1.0, 2 ** 31 - 2048), (1e4, 1_000_000), (1e6, 1_000_000), (1e6, 2 ** 31 - 2048)))
def test_keys_at_far_angles(dtype, layout, rot, freq, start):
    """Keys are held as the rounding of the exact rotation by the angle p f, a product in 64 bits,
    however many turns that is."""
    Hkv, T, d, page = 8, 512, 128, 256
    W = (start + T) // page + 1
    table = torch.full((1, W), -1, dtype=torch.int32)
    table[0, start // page:] = torch.arange(W - start // page)
    cache = kia.new_cache4(8, Hkv, page, d)
    plan = kia.RotaryPlan(torch.linspace(freq / 2, freq, rot // 2, dtype=torch.float64, device="cuda"), layout)
    k = draw((1, Hkv, T, d), dtype, 11, 2.0)
    kia.cache4_append(k, k, k, cache, table.cuda(), ints(start), plan)
    got = kia.cache4_read(cache, table.cuda(), ints(start), T, torch.float32)[0]
    want = ref.rotary(k, plan.freq, layout, plan.factor, torch.arange(start, start + T, device="cuda")[None])[0]
    assert torch.equal(got.double(), ref.held(want))
