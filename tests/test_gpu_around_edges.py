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
