"""Inputs whose tangents or whose trace a call would lose are refused (no GPU needed: the
refusal comes before that of host tensors)."""
import pytest

torch = pytest.importorskip("torch")

import torch.autograd.forward_ad as ad  # noqa: E402

import paper_2609_33591_amd as kia  # noqa: E402


def calls():
    """{name: (call of one tensor, the tensor)}; the others' arguments are ordinary."""
    q, k = torch.zeros(2, 4, 8, 64), torch.zeros(2, 2, 8, 64)
    lse = torch.zeros(2, 4, 8)
    plan = kia.rotary_plan(64, device="cpu")
    cache = kia.new_cache4(3, 2, 16, 64, device="cpu")
    table, one = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    return {
        "rotary q": (lambda x: kia.rotary(x, k, plan)[0], q),
        "rotary k": (lambda x: kia.rotary(q, x, plan)[0], k),
        "k_interval_attention q": (lambda x: kia.k_interval_attention(x, q, q), q),
        "k_interval_attention v": (lambda x: kia.k_interval_attention(q, q, x, rotary=plan), q),
        "window_attention q": (lambda x: kia.window_attention(x, k, k, 4), q),
        "window_attention v": (lambda x: kia.window_attention(q, k, x, 4), k),
        "window_attention rotary": (lambda x: kia.window_attention(q, k, x, 4, rotary=plan), k),
        "window_forward": (lambda x: kia.window_forward(q, x, k, 4)[0], k),
        "window_backward": (lambda x: kia.window_backward(q, k, k, q, x, lse, 4)[0], q),
        "cache4_write": (lambda x: kia.cache4_write(k, x, cache, table, one), k),
        "cache4_attention": (lambda x: kia.cache4_attention(x, cache, table, one), q),
    }


@pytest.mark.parametrize("name", calls())
def test_tangents_are_refused(name):
    fn, x = calls()[name]
    with ad.dual_level():
        with pytest.raises(kia.KiaError, match="tangent"):
            fn(ad.make_dual(x, torch.ones_like(x)))
        # tensors without one pass, also beside others that have one
        with pytest.raises(kia.KiaError, match="device tensors"):
            fn(x)
    with pytest.raises(kia.KiaError, match="device tensors"):
        fn(x)


@pytest.mark.filterwarnings("ignore::DeprecationWarning")
@pytest.mark.parametrize("name", calls())
def test_traces_are_refused(name):
    fn, x = calls()[name]
    with pytest.raises(kia.KiaError, match="cannot be traced"):
        torch.jit.trace(fn, (x,))
