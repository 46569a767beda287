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
