"""The operators that serve from the 4-bit cache refuse inputs whose tangents or whose trace a call
would lose (no GPU needed: the refusal comes before that of host tensors)."""
import pytest

torch = pytest.importorskip("torch")

import torch.autograd.forward_ad as ad  # noqa: E402

import paper_2609_33591_amd as kia  # noqa: E402


def calls():
    """{name: (call of one tensor, the tensor)}; the others' arguments are ordinary."""
    q, k = torch.zeros(2, 4, 1, 64), torch.zeros(2, 2, 1, 64)
    plan = kia.rotary_plan(64, device="cpu")
    cache = kia.new_cache4(3, 2, 16, 64, device="cpu")
    bounds = kia.new_bounds4(cache)
    table, one = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    pages = torch.zeros(2, 2, 1, 3, dtype=torch.int32)
    return {
        "append q": (lambda x: kia.cache4_append(x, k, k, cache, table, one, plan), q),
        "append k": (lambda x: kia.cache4_append(q, x, k, cache, table, one, plan, bounds=bounds), k),
        "append v": (lambda x: kia.cache4_append(q, k, x, cache, table, one, plan, one), k),
        "select": (lambda x: kia.cache4_select(x, cache, bounds, table, one, 3), q),
        "attention over pages": (lambda x: kia.cache4_attention(x, cache, table, one, pages=pages), q),
        "attention behind shared": (lambda x: kia.cache4_attention(x, cache, table, one, shared=32), q),
    }


@pytest.mark.parametrize("name", calls())
def test_tangents_are_refused(name):
    fn, x = calls()[name]
    with ad.dual_level():
        with pytest.raises(kia.KiaError, match="tangent"):
            fn(ad.make_dual(x, torch.ones_like(x)))
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


@pytest.mark.filterwarnings("ignore::DeprecationWarning")
def test_bounds_in_a_trace_are_refused():
    cache = kia.new_cache4(3, 2, 16, 64, device="cpu")
    bounds, table, one = kia.new_bounds4(cache), torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)

    def fn(x):
        kia.cache4_bounds(cache, bounds, table, one, one)
        return x

    with pytest.raises(kia.KiaError, match="cannot be traced"):
        torch.jit.trace(fn, (torch.zeros(1),))
