"""Positions of shape [1, T], the same for every sequence of a batch."""
import pytest

torch = pytest.importorskip("torch")

import paper_2609_33591_amd as kia  # noqa: E402
from paper_2609_33591_amd import around  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("B", (1, 3))
def test_one_row_of_positions_for_a_batch(dtype, B, monkeypatch):
    g = torch.Generator().manual_seed(1)
    q, k = (torch.randn(B, h, 33, 64, generator=g).to(dtype).cuda() for h in (4, 2))
    plan = kia.rotary_plan(48, layout="interleaved")
    pos = torch.randint(-9, 5000, (33,), generator=g, dtype=torch.int32).cuda()
    want = kia.rotary(q, k, plan, pos)
    y, z = torch.empty_like(q), torch.empty_like(k)
    kia.kia_rotary(q, k, y, z, plan, pos[None])
    assert torch.equal(y, want[0]) and torch.equal(z, want[1])
    o = kia.window_attention(q, k, k, 7, rotary=plan, positions=pos)
    for _ in range(2):  # by the C module, and without it
        for p in (pos[None], pos.expand(B, 33).contiguous()):
            assert all(torch.equal(a, b) for a, b in zip(kia.rotary(q, k, plan, p), want))
        assert torch.equal(kia.window_attention(q, k, k, 7, rotary=plan, positions=pos[None]), o)
        monkeypatch.setattr(around, "_fast", lambda: type("None_", (), {
            "rotary": lambda *a: None, "window_forward": lambda *a: None}))
    x = q.clone().requires_grad_()
    monkeypatch.undo()
    dq, = torch.autograd.grad(kia.rotary(x, None, plan, pos[None])[0], x, q)
    assert torch.equal(dq, kia.rotary(q, None, plan, pos, back=True)[0])


def test_other_shapes_are_refused():
    q, plan = torch.zeros(3, 2, 8, 64, device="cuda"), kia.rotary_plan(64)
    for shape in ((2, 8), (1, 7), (3, 1), (1, 1, 8), (8, 1), (1, 3, 8), (0, 8)):
        with pytest.raises(kia.KiaError, match="positions has shape"):
            kia.rotary(q, None, plan, torch.zeros(shape, dtype=torch.int32, device="cuda"))
