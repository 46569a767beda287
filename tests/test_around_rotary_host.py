"""Rotary positions without keys look at no number of key heads (no GPU needed)."""
import pytest

torch = pytest.importorskip("torch")

from tests.test_around_host import NULL, SHAPE, lib, rotary  # noqa: E402,F401


def test_key_heads_without_keys(lib):  # noqa: F811
    for Hkv in (0, -1, 65535, 1 << 30, -(1 << 31)):
        # (the missing output stops the call)
        assert rotary(lib, q_out=None, k=None, k_out=None, Hkv=Hkv) == NULL
        assert rotary(lib, q_out=None, k=None, k_out=None, Hkv=Hkv, H=65536) == SHAPE
    assert rotary(lib, q_out=None, Hkv=65533) == NULL
    assert rotary(lib, q_out=None, Hkv=65534) == SHAPE
