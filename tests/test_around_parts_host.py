"""The windowed backward cuts its key blocks into a bounded number of parts (no GPU
needed): what its workspace is sized for and its launches count on."""
import ctypes
import math
import random

import pytest

torch = pytest.importorskip("torch")

from tests.test_around_host import lib  # noqa: E402,F401


def slots(lib, B, H, Hkv, T, d, window, sinks):  # noqa: F811
    """Partial sums of the key blocks of all key heads, by the workspace: D of every row,
    then 64 rows of dK and of dV for each."""
    n = ctypes.c_size_t(0)
    assert lib.kia_window_ws_bytes(B, H, Hkv, T, d, window, sinks, ctypes.byref(n)) == 0
    rest = n.value - (B * H * T * 4 + 255) // 256 * 256
    assert rest >= 0 and rest % (2 * 64 * d * 4) == 0
    return rest // (2 * 64 * d * 4)


def test_parts_of_key_blocks(lib):  # noqa: F811
    rng = random.Random(5)
    shapes = [(1, 2, 1, 3348, 64, 166, 1 << 30), (1, 9, 3, 1553, 64, 111, 1553), (1, 1, 1, 1 << 24, 128, 1, 1 << 24)]
    for _ in range(20000):
        Hkv, B, T = (int(math.exp(rng.uniform(0, math.log(x)))) for x in (60, 20, 1 << 17))
        shapes.append((B, Hkv * rng.randint(1, 8), Hkv, T, rng.choice((16, 32, 64, 128)),
                       int(math.exp(rng.uniform(0, 12))), rng.choice((0, 1, 100, T // 3, T))))
    most = 0
    for s in shapes:
        B, _, Hkv, T = s[:4]
        more = slots(lib, *s) - B * Hkv * ((T + 63) // 64)
        assert more < 2816, s
        most = max(most, more)
    assert most > 2560  # (the first shapes pass it)
