"""The windowed attention's lse of another shape than [B, heads, T] is refused (no GPU
needed: the refusal comes before that of host tensors)."""
import pytest

torch = pytest.importorskip("torch")

import paper_2609_33591_amd as kia  # noqa: E402


@pytest.mark.parametrize("shape", ((2, 8, 4), (2, 4, 9), (2, 5, 8), (3, 4, 8), (64,), (2, 4, 8, 1), (1, 4, 8)))
def test_lse_of_another_shape(shape):
    q, k = torch.zeros(2, 4, 8, 64), torch.zeros(2, 2, 8, 64)
    lse = torch.zeros(shape)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    for fn in (lambda: kia.window_backward(q, k, k, q, q, lse, 4),
               lambda: kia.kia_window_fwd(q, k, k, torch.empty_like(q), lse, 4),
               lambda: kia.kia_window_bwd(q, k, k, q, q, lse, ws[-(ws.data_ptr() % 256) % 256:], *map(
                   torch.empty_like, (q, k, k)), 4)):
        with pytest.raises(kia.KiaError, match="lse has shape"):
            fn()


@pytest.mark.parametrize("lse", (torch.zeros(2, 8, 4).transpose(1, 2), torch.zeros(2, 4, 8, dtype=torch.float64)))
def test_lse_of_another_layout_or_type(lse):
    q, k = torch.zeros(2, 4, 8, 64), torch.zeros(2, 2, 8, 64)
    with pytest.raises(kia.KiaError, match="lse must be a contiguous torch.float32"):
        kia.window_backward(q, k, k, q, q, lse, 4)
    with pytest.raises(kia.KiaError, match="lse must be a contiguous torch.float32"):
        kia.kia_window_fwd(q, k, k, torch.empty_like(q), lse, 4)
