"""The error of bfloat16 calls as a whole, by the 2-norm over an output: the bounds of single
values elsewhere hold for worst cases, and would not show a kernel that is worse than it
has to be everywhere.

With r the error of an output's own rounding alone (of the exact values, in the same
norm): weights and score gradients are sums' factors, rounded as the outputs are. Over
random values the terms of such a sum are as good as independent, so its roundings add
an error of r times the sum's own norm: together sqrt(2) r. The goal is 1.5 r. A factor
in two pieces (2^-16) adds nothing: 1.25 r there."""
import pytest

torch = pytest.importorskip("torch")

import paper_2609_33591_amd as kia  # noqa: E402
from tests import around_reference as ref  # noqa: E402
from tests.test_gpu_cache4 import draw, filled, ints  # noqa: E402
from tests.test_gpu_window import inputs  # noqa: E402

pytestmark = pytest.mark.gpu


def share(got, want):
    """The error of `got` over that of the rounding of `want`."""
    err = (got.double() - want).norm()
    return float(err / (want.to(got.dtype).double() - want).norm())


@pytest.mark.parametrize("B,H,Hkv,T,d,window,sinks", [
    (1, 2, 1, 4000, 16, 217, 100), (1, 2, 1, 4000, 32, 217, 100), (1, 2, 1, 4000, 64, 217, 100),
    (1, 2, 1, 2000, 128, 512, 4),
    # rows of few keys, where D from the rounded output would pass all other errors
    (2, 4, 2, 900, 128, 2, 0), (2, 4, 2, 900, 16, 3, 1), (2, 4, 2, 900, 64, 30, 2),
    # the grids of four groups of rows
    (8, 64, 16, 300, 128, 2, 0), (8, 104, 26, 300, 32, 217, 0)])
def test_window(B, H, Hkv, T, d, window, sinks):
    q, k, v, g = inputs(B, H, Hkv, T, d, torch.bfloat16, seed=300)
    o, lse = kia.window_forward(q, k, v, window, sinks)
    grads = kia.window_backward(q, k, v, o, g, lse, window, sinks)
    # (of the large grids one key head and its queries)
    b, h = (B, Hkv) if B * H < 64 else (1, 1)
    part = lambda x: x[:b, :h * x.shape[1] // Hkv]  # noqa: E731
    want = ref.window(*(part(x).contiguous() for x in (q, k, v)), window, sinks, None, part(g).contiguous())
    for name, x in zip(("o", "dq", "dk", "dv"), (o, *grads)):
        s = share(part(x), want[name][0])
        assert s <= (1.25 if name == "dq" and d <= 32 else 1.5), (name, s)


@pytest.mark.parametrize("op", (dict(recon="softmax"), dict(recon="lerp", calib="fwm", K=4, tau=8.0),
                                dict(recon="lerp", calib="minmax", K=16)), ids=lambda o: "-".join(map(str, o.values())))
@pytest.mark.parametrize("H,T", ((4, 1), (16, 2)))
def test_cached(op, H, T):
    lengths = (3000, 200, 900)
    cache, table, k, v = filled(lengths, 4, 64, 64, torch.bfloat16, 310)
    q = draw((3, H, T, 64), torch.bfloat16, 314)
    o = kia.cache4_attention(q, cache, table, ints(*lengths), **op)
    want = torch.stack([ref.cached(q[b], k[b, :, :n], v[b, :, :n], n, **op)[0] for b, n in enumerate(lengths)])
    s = share(o, want)
    assert s <= 1.5, s
