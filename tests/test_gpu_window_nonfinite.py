"""Windowed attention on the device where infinities and NaNs stand in rows that are
seen: what they reach goes by the definition, not by the tile that a row or the end of
a sequence falls in. Everything else is compared bit for bit with a call of finite
values in their place that has the same weights."""
import itertools
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2609_33591_amd as kia  # noqa: E402
from tests.test_gpu_window import inputs  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = (torch.float32, torch.bfloat16)
# grids of two and of four groups of rows in a workgroup
GRIDS = ((1, 2, 1), (2, 208, 8))


def both(q, k, v, g, window, sinks, lengths=None):
    o, lse = kia.window_forward(q, k, v, window, sinks, lengths)
    return (o, lse, *kia.window_backward(q, k, v, o, g, lse, window, sinks, lengths))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", (16, 64, 128))
@pytest.mark.parametrize("grid", GRIDS)
@pytest.mark.parametrize("bad", (math.nan, math.inf, -math.inf))
def test_rows_behind_a_sequence_stay_zero(dtype, d, grid, bad):
    """The last token of a sequence in the middle of a tile is not finite: what is behind
    the end is 0 all the same."""
    B, H, Hkv = grid
    T, n = 150, 77
    lengths = torch.full((B,), n, dtype=torch.int32, device="cuda")
    for which in range(4):
        x = inputs(B, H, Hkv, T, d, dtype, seed=200)
        x[which][:, :, n - 1, 3] = bad
        o, lse, *grads = both(*x, 40, 2, lengths)
        for y in (o, *grads):
            assert bool((y[:, :, n:] == 0).all()), which
        assert bool((lse[:, :, n:] == -math.inf).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", (16, 64, 128))
@pytest.mark.parametrize("grid", GRIDS)
def test_rows_of_no_weight_are_zero(dtype, d, grid):
    """A query whose every score is -infinity has o = 0, lse = -infinity and dq = 0,
    whatever the values that it sees hold."""
    B, H, Hkv = grid
    T = 150
    q, k, v, g = inputs(B, H, Hkv, T, d, dtype, seed=230)
    k[..., 3] = k[..., 3].abs() + 0.5
    q[:, :, 100, 3] = -math.inf
    for window, sinks in ((T, 0), (40, 2)):
        for bad in (math.inf, math.nan):
            y = v.clone()
            y[:, :, 80, 1] = bad
            o, lse, dq, *_ = both(q, k, y, g, window, sinks)
            assert bool((o[:, :, 100] == 0).all()) and bool((dq[:, :, 100] == 0).all())
            assert bool((lse[:, :, 100] == -math.inf).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", (16, 64, 128))
@pytest.mark.parametrize("grid", GRIDS)
def test_rows_of_no_weight_add_nothing(dtype, d, grid):
    """A query whose every score is -infinity adds nothing to dk and dv, whatever its dO
    holds, and changes no other row."""
    B, H, Hkv = grid
    T = 150
    q, k, v, g = inputs(B, H, Hkv, T, d, dtype, seed=210)
    k[..., 3] = k[..., 3].abs() + 0.5
    for at in (0, 31, 70, 149):
        for window, sinks in ((T, 0), (40, 2)):
            # a row with dO = 0 adds nothing to dk and dv either
            g0 = g.clone()
            g0[:, :, at] = 0
            want = both(q, k, v, g0, window, sinks)
            x, bad = q.clone(), g.clone()
            x[:, :, at, 3] = -math.inf
            for value in (1.0, math.nan, math.inf):
                bad[:, :, at, 1] = value
                o, lse, dq, dk, dv = both(x, k, v, bad, window, sinks)
                rest = torch.arange(T, device="cuda") != at
                assert bool((o[:, :, at] == 0).all()) and bool((dq[:, :, at] == 0).all())
                assert bool((lse[:, :, at] == -math.inf).all())
                for got, to in zip((o, lse, dq), want):
                    assert torch.equal(got[:, :, rest], to[:, :, rest])
                assert torch.equal(dk, want[3]) and torch.equal(dv, want[4])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", (16, 64, 128))
@pytest.mark.parametrize("n", (65, 77, 97, 150))
def test_keys_of_no_weight_beside_the_end(dtype, d, n):
    """A key whose scores are all -infinity has no gradient, also where rows behind the
    end of its sequence share its tile."""
    T = 150
    q, k, v, g = inputs(2, 2, 1, T, d, dtype, seed=240)
    q[..., 3] = q[..., 3].abs() + 0.5
    k[:, :, 40, 3] = -math.inf
    lengths = torch.full((2,), n, dtype=torch.int32, device="cuda")
    for window, sinks in ((T, 0), (70, 0), (30, 2)):
        *_, dk, dv = both(q, k, v, g, window, sinks, lengths)
        assert bool((dk[:, :, 40] == 0).all()) and bool((dv[:, :, 40] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", (16, 64, 128))
@pytest.mark.parametrize("grid", GRIDS)
def test_keys_of_scores_of_minus_infinity(dtype, d, grid):
    """A key whose scores are all -infinity has weight 0 as one whose scores are far below
    the others': the same outputs and gradients, but for dq, which is NaN in the channel
    where 0 meets the infinity; in every kind of tile, and beside the end of a sequence."""
    B, H, Hkv = grid
    T = 150
    q, k, v, g = inputs(B, H, Hkv, T, d, dtype, seed=220)
    q[..., 3] = q[..., 3].abs() + 0.5
    i = torch.arange(T, device="cuda")
    for at, n, (window, sinks) in itertools.product((0, 5, 40, 63, 64), (65, 77, 96, 97, 128, T),
                                                    ((T, 0), (70, 0), (30, 2))):
        lengths = torch.full((B,), n, dtype=torch.int32, device="cuda")
        low, none = k.clone(), k.clone()
        low[:, :, at, 3] = -2.0 ** 15  # (scores below -2^10: weight 0 in fp32)
        none[:, :, at, 3] = -math.inf
        want, got = (both(q, x, v, g, window, sinks, lengths) for x in (low, none))
        see = (i >= at) & ((i - at < window) | (at < sinks)) & (i < n)
        # the first row sees no other key than the first: no weight, where the finite
        # score has all of it
        alone = (i == 0) & (at == 0)
        what = f"key {at}, {n} tokens, window {window}"
        for a, b in zip(got[:2], want[:2]):
            assert torch.equal(a[:, :, ~alone], b[:, :, ~alone]), what
        dq, see = got[2], see & ~alone
        assert bool((got[0][:, :, alone] == 0).all()) and bool((dq[:, :, alone] == 0).all()), what
        assert bool(torch.isnan(dq[:, :, see][..., 3]).all()), what
        dq[..., 3] = torch.where(see, want[2][..., 3], dq[..., 3])
        assert torch.equal(dq[:, :, ~alone], want[2][:, :, ~alone]), what
        if at == 0:
            g0 = g.clone()
            g0[:, :, 0] = 0
            want = both(q, low, v, g0, window, sinks, lengths)
        assert torch.equal(got[3], want[3]), what
        assert torch.equal(got[4], want[4]), what
        assert bool((got[3][:, :, at] == 0).all()) and bool((got[4][:, :, at] == 0).all()), what
