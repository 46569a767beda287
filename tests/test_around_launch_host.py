"""Calls of more workgroups than a launch can have are refused on the host."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from tests.test_around_host import SHAPE, cache, lib, rotary, window  # noqa: E402,F401


def test_more_workgroups_than_a_launch_has(lib):  # noqa: F811
    # a workgroup for each sequence of one token; one fewer is stopped by another check
    assert rotary(lib, B=1 << 24, T=1) == SHAPE
    assert rotary(lib, B=(1 << 24) - 1, T=1, q=None) != SHAPE
    for fwd in (True, False):
        assert window(lib, fwd, B=1 << 23, H=2, T=1) == SHAPE
        assert window(lib, fwd, B=(1 << 23) - 4096, H=2, T=64, x=None, lse=None) != SHAPE
        assert window(lib, fwd, B=1 << 20, H=1 << 3, Hkv=1, T=1 << 10) == SHAPE
    for op in ("write", "read"):
        assert cache(lib, op, B=1 << 22, Hkv=2, H=2, T=1) == SHAPE
        assert cache(lib, op, B=(1 << 22) - 1, Hkv=2, H=2, T=1, starts=None) != SHAPE
    assert cache(lib, "attn", B=1 << 23, Hkv=2, H=2, T=1) == SHAPE
    # (few key heads, many rows, keys in several parts: the join has a workgroup a row)
    assert cache(lib, "attn", B=1 << 14, Hkv=1, H=1, T=1 << 10, width=1 << 10, page=16) == SHAPE
    n = ctypes.c_size_t(1)
    assert lib.kia_cache4_ws_bytes(16, 1, 1 << 24, 1, 1, 1, 64, 0, 0, ctypes.byref(n)) == SHAPE
