"""The operators around K-interval attention: rotary positions, softmax attention
with a sliding window and visible first tokens, a paged key/value cache in 4
bits, and attention of new tokens over it: over all of a text, over the pages that
their bounds select, or behind tokens that a batch shares.

The ``kia_*`` functions carry the names of the C-ABI entry points of
``include/kia.h`` and only marshal arguments, on buffers of the caller's; the
others allocate what they return. Tensors are [B, heads, T, d], float32 or
bfloat16 throughout a call, with contiguous rows and any other strides (a
projection's [B, T, heads, d] transposed needs no copy).
"""
from __future__ import annotations

import ctypes
import functools
import math
from dataclasses import dataclass

import paper_2609_33591_amd as _kia

KiaError = _kia.KiaError

# rotary layouts: which channels make a pair
LAYOUT = {"half": 0, "interleaved": 1}


class View(ctypes.Structure):
    """kia_view: data and the strides of B, heads and T in elements."""
    _fields_ = [("data", ctypes.c_void_p), ("sb", ctypes.c_int64), ("sh", ctypes.c_int64),
                ("st", ctypes.c_int64)]


def declare(lib):
    """Argument types of the entry points (called by load())."""
    V, P, I, F, S = (ctypes.POINTER(View), ctypes.c_void_p, ctypes.c_int, ctypes.c_float,
                     ctypes.POINTER(ctypes.c_size_t))
    for name, types in (
            ("kia_rotary", [V] * 4 + [P, ctypes.c_int64, I, P, F] + [I] * 9 + [P]),
            ("kia_window_ws_bytes", [I] * 7 + [S]),
            ("kia_window_fwd", [V] * 4 + [P, P] + [I] * 8 + [P]),
            ("kia_window_bwd", [V] * 5 + [P, P, P] + [V] * 3 + [I] * 8 + [P]),
            ("kia_cache4_bytes", [I] * 4 + [S]),
            ("kia_cache4_write", [V, V, P, I, I, P, I, P, P] + [I] * 5 + [P]),
            ("kia_cache4_read", [P, I, I, P, I, P, P, V, V] + [I] * 5 + [P]),
            ("kia_cache4_ws_bytes", [I] * 9 + [S]),
            ("kia_cache4_attn", [V, V, P, I, I, P, I, P, P] + [I] * 7 + [F] + [I] * 4 + [P]),
            ("kia_cache4_append", [V] * 4 + [P, P, I, I, P, I, P, P, P, F] + [I] * 8 + [P]),
            ("kia_cache4_bounds", [P, P, I, I, P, I, P, P, I, I, I, P]),
            ("kia_cache4_select_ws_bytes", [I] * 7 + [S]),
            ("kia_cache4_select", [V, P, I, I, P, I, P, P, P] + [I] * 9 + [P]),
            ("kia_cache4_pages_ws_bytes", [I] * 8 + [S]),
            ("kia_cache4_attn_pages", [V, V, P, I, I, P, I, P, P, I, P] + [I] * 7 + [F, I, I, P]),
            ("kia_cache4_shared_ws_bytes", [I] * 8 + [S]),
            ("kia_cache4_attn_shared", [V, V, P, I, I, P, I, P, I, P] + [I] * 7 + [F, I, I, P])):
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = types, I


# ---- checks -------------------------------------------------------------------
# (What goes by shapes, strides and types alone is looked up: a serving loop repeats it
# call after call, and a call for a token is as long as its host work.)
@functools.lru_cache(maxsize=4096)
def _fit(shape, stride, dtype):
    """The strides of B, heads and T of a tensor's layout, or why the kernels cannot
    take it."""
    import torch
    if len(shape) != 4:
        return f"must be [B, heads, T, d], got shape {tuple(shape)}"
    if dtype not in (torch.float32, torch.bfloat16):
        return f"must be float32 or bfloat16, got {dtype}"
    B, H, T, d = shape
    sb, sh, st, sd = stride
    unit = 4 if dtype == torch.float32 else 8
    if sd != 1:
        return "has channels that are not contiguous"
    if T > 1 and (st < d or st % unit or st > 1 << 22):
        return f"has rows {st} elements apart"
    if (H > 1 and sh % unit) or (B > 1 and sb % unit):
        return "is not 16-byte aligned"
    return sb, sh, st


@functools.lru_cache(maxsize=4096)
def _dense(shape):
    B, H, T, d = shape
    return H * T * d, T * d, d


class _Like:
    """What every tensor of a call has in common: the first one's type and device,
    batch, tokens and channels."""
    __slots__ = ("shape", "dtype", "device", "code")

    def __init__(self, name, t):
        import torch
        if t.dim() != 4:
            raise KiaError(f"{name} must be [B, heads, T, d], got shape {tuple(t.shape)}")
        self.shape, self.dtype, self.device = t.shape, t.dtype, t.device
        if self.dtype == torch.float32:
            self.code = 0
        elif self.dtype == torch.bfloat16:
            self.code = 1
        else:
            raise KiaError(f"tensors must be float32 or bfloat16, got {self.dtype}")

    def view(self, name, t, heads=None, out=False):
        """A tensor as a kia_view, with `heads` heads (None: the first one's)."""
        want = self.shape if heads is None else (self.shape[0], heads, self.shape[2], self.shape[3])
        if t.shape != want:
            raise KiaError(f"{name} has shape {tuple(t.shape)}, expected {tuple(want)}")
        if t.dtype != self.dtype:
            raise KiaError(f"{name} has dtype {t.dtype}, expected {self.dtype}")
        if t.device != self.device:
            raise KiaError(f"{name} is on {t.device}, expected {self.device}")
        fit, ptr = _fit(t.shape, t.stride(), t.dtype), t.data_ptr()
        if type(fit) is str or ptr % 16:
            raise KiaError(f"{name} {fit if type(fit) is str else 'is not 16-byte aligned'}")
        if out and ((want[0] > 1 and fit[0] == 0) or (want[1] > 1 and fit[1] == 0)):
            raise KiaError(f"{name} is written to and must not be expanded")
        return View(ptr, *fit)

    def take(self, name, t, heads=None):
        """view() of a tensor to be read, or of a contiguous copy where the kernels
        cannot take its layout (kept alive by the caller: (tensor, view))."""
        import torch
        want = self.shape if heads is None else (self.shape[0], heads, self.shape[2], self.shape[3])
        if t.shape == want and t.dtype == self.dtype and t.device == self.device:
            fit, ptr = _fit(t.shape, t.stride(), t.dtype), t.data_ptr()
            if type(fit) is tuple and ptr % 16 == 0:
                return t, View(ptr, *fit)
            t = t.clone(memory_format=torch.contiguous_format)
        return t, self.view(name, t, heads)


def _new(ref):
    """A new contiguous tensor of ref's shape and its view."""
    import torch
    t = torch.empty_like(ref, memory_format=torch.contiguous_format)
    return t, View(t.data_ptr(), *_dense(t.shape))


def _heads(q, k):
    if q.dim() != 4 or k.dim() != 4:
        raise KiaError(f"tensors must be [B, heads, T, d], got {tuple(q.shape)}, {tuple(k.shape)}")
    return k.shape[1]


def _ints(name, t, shape, device):
    """Device pointer of a contiguous int32 tensor (None: NULL)."""
    import torch
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype != torch.int32:
        raise KiaError(f"{name} must be an int32 tensor")
    if t.shape != shape:
        raise KiaError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.device != device:
        raise KiaError(f"{name} is on {t.device}, expected {device}")
    if not t.is_contiguous():
        raise KiaError(f"{name} must be contiguous")
    return t.data_ptr()


def _buffer(name, t, dtype, least, device, align):
    if t.dtype != dtype or not t.is_contiguous() or t.device != device:
        raise KiaError(f"{name} must be a contiguous {dtype} tensor on {device}")
    if t.numel() < least:
        raise KiaError(f"{name} holds {t.numel()} elements, the call needs {least}")
    ptr = t.data_ptr()
    if ptr % align:
        raise KiaError(f"{name} must be {align}-byte aligned")
    return ptr


def _call(fn, device, stream, *args):
    """The call on `device`, on its current stream if none is given."""
    import torch
    if device.type != "cuda":
        raise KiaError("libkia takes device tensors only")
    if stream is not None and getattr(stream, "device", device) != device:
        raise KiaError(f"the stream is on {stream.device}, the tensors on {device}")
    if torch._C._cuda_getDevice() == device.index:
        rc = fn(*args, _kia._stream(stream))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, _kia._stream(stream))
    if rc:
        _kia._check(rc)


def _int(name, x, low):
    if type(x) is not int or not low <= x < 1 << 31:
        raise KiaError(f"{name} must be an integer of at least {low}, got {x!r}")
    return x


_modes = []  # torch.autograd.forward_ad and torch's tracing state, looked up once


def _eager(*tensors):
    """Refuses what a call would leave out without a word, since the kernels see data
    alone: forward-mode derivatives of its inputs (their tangents), and its place in a
    trace."""
    if not _modes:
        import torch
        _modes.extend((torch.autograd.forward_ad, torch._C._get_tracing_state))
    ad, trace = _modes
    if ad._current_level < 0 and trace() is None:
        return
    if any(hasattr(x, "requires_grad") and ad.unpack_dual(x).tangent is not None for x in tensors):
        raise KiaError("libkia has no forward-mode derivatives: an input has a tangent")
    if trace() is not None:
        raise KiaError("libkia's calls cannot be traced")


# The allocating calls go through csrc/kia_host.c where every argument is as the kernels
# take it (a call for one token 9 us instead of 14); it returns None where one is not, and
# the code below then copies what needs copying, or says what is wrong.
@functools.lru_cache(maxsize=1)
def _fast():
    import torch
    lib = _kia.load()
    try:
        from . import _host
    except ImportError as e:
        raise KiaError(f"the binding's C module is missing: run paper_2609_33591_amd.build ({e})")
    _host.bind(torch, _kia._check, {
        n: ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in (
            "kia_rotary", "kia_window_fwd", "kia_window_ws_bytes", "kia_window_bwd",
            "kia_cache4_write", "kia_cache4_read", "kia_cache4_ws_bytes", "kia_cache4_attn",
            "kia_cache4_append", "kia_cache4_select_ws_bytes", "kia_cache4_select",
            "kia_cache4_pages_ws_bytes", "kia_cache4_attn_pages", "kia_cache4_shared_ws_bytes",
            "kia_cache4_attn_shared")})
    return _host


# ---- rotary positions -----------------------------------------------------------
@dataclass(eq=False)
class RotaryPlan:
    """Frequencies (float64 [rot / 2] on the device, radians per position), the
    layout of a pair ("half": channels n and n + rot/2; "interleaved": 2n and
    2n + 1) and the factor of the rotated channels."""
    freq: object
    layout: str = "half"
    factor: float = 1.0


def rotary_plan(rot, base=10000.0, layout="half", scaling="none", stretch=1.0, original=None,
                turns=(1.0, 32.0), device="cuda"):
    """The plan of `rot` rotated channels with frequencies base^(-2n / rot).

    For contexts `stretch` times as long as trained on (`original` positions):
    "linear" divides every frequency by it; "base" raises the base so that the
    slowest pair is stretched by it and the fastest keeps its frequency;
    "parts" divides those of pairs that turn fewer than turns[0] times over the
    original context, keeps those of more than turns[1] and blends between,
    with factor 0.1 ln(stretch) + 1."""
    import torch
    n = _int("rot", rot, 2) // 2
    if rot % 2:
        raise KiaError(f"rot must be even, got {rot}")
    if layout not in LAYOUT:
        raise KiaError(f"layout must be one of {sorted(LAYOUT)}, got {layout!r}")
    if scaling not in ("none", "linear", "base", "parts"):
        raise KiaError(f"scaling must be none, linear, base or parts, got {scaling!r}")
    if not base > 0 or not stretch > 0:
        raise KiaError("base and stretch must be positive")
    factor = 1.0
    if scaling == "base":
        base = base * stretch ** (n / max(1, n - 1))
    freq = [base ** (-i / n) for i in range(n)]
    if scaling == "linear":
        freq = [f / stretch for f in freq]
    if scaling == "parts":
        if original is None or not original > 0 or not turns[0] < turns[1]:
            raise KiaError("parts needs original > 0 and turns[0] < turns[1]")
        for i, f in enumerate(freq):
            t = original * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (t - turns[0]) / (turns[1] - turns[0])))
            freq[i] = f / stretch * (1 - keep) + f * keep
        factor = 0.1 * math.log(stretch) + 1.0
    return RotaryPlan(torch.tensor(freq, dtype=torch.float64, device=device), layout, factor)


def _rotary_call(like, views, Hkv, plan, positions, back, stream=None):
    import torch
    B, H, T, d = like.shape
    freq = plan.freq
    if freq.dim() != 1 or not 2 <= 2 * freq.shape[0] <= d:
        raise KiaError(f"a plan's frequencies must be one to {d // 2} in one dimension for heads of "
                       f"{d} channels, got shape {tuple(freq.shape)}")
    fp = _buffer("the plan's frequencies", freq, torch.float64, 1, like.device, 8)
    first, ptr, sb = 0, None, 0
    if isinstance(positions, torch.Tensor):
        if positions.dim() == 1:
            ptr = _ints("positions", positions, (T,), like.device)
        elif positions.dim() == 2 and positions.shape[0] == 1:
            ptr = _ints("positions", positions, (1, T), like.device)
        else:
            ptr, sb = _ints("positions", positions, (B, T), like.device), T
    elif positions is not None:
        if type(positions) is not int or not -(1 << 31) <= positions < 1 << 31:
            raise KiaError(f"positions must be an int32 tensor or an integer, got {positions!r}")
        first = positions
    if plan.layout not in LAYOUT:
        raise KiaError(f"layout must be one of {sorted(LAYOUT)}, got {plan.layout!r}")
    _call(_kia.load().kia_rotary, like.device, stream, *views, ptr, sb, first, fp,
          float(plan.factor), LAYOUT[plan.layout], 1 if back else 0, B, H, Hkv, T, d,
          2 * freq.shape[0], like.code)


def kia_rotary(q, k, q_out, k_out, plan, positions=None, back=False, stream=None):
    """Rotates q (and k; None: only q) into q_out (k_out), which may be q and k.
    positions: int32 [B, T], or [1, T] or [T] for every sequence, the first position
    as an integer, or None (0). back: by the negative angle, the gradient of the rotation."""
    like = _Like("q", q)
    views, Hkv = [like.view("q", q), like.view("q_out", q_out, out=True), None, None], 0
    if k is not None:
        Hkv = _heads(q, k)
        views[2:] = like.view("k", k, Hkv), like.view("k_out", k_out, Hkv, True)
    _rotary_call(like, views, Hkv, plan, positions, back, stream)


def _rotated(q, k, plan, positions, back):
    made = _fast().rotary(q, k, plan.freq, positions, LAYOUT.get(plan.layout, -1), plan.factor,
                          1 if back else 0)
    if made is not None:
        return made
    like = _Like("q", q)
    q, vq = like.take("q", q)
    q_out, vo = _new(q)
    if k is None:
        _rotary_call(like, (vq, vo, None, None), 0, plan, positions, back)
        return q_out, None
    Hkv = _heads(q, k)
    k, vk = like.take("k", k, Hkv)
    k_out, vy = _new(k)
    _rotary_call(like, (vq, vo, vk, vy), Hkv, plan, positions, back)
    return q_out, k_out


@functools.lru_cache(maxsize=1)
def _rotary_function():
    import torch

    class Rotary(torch.autograd.Function):
        """The rotation is linear: its gradient is the rotation back (which keeps
        the plan and the positions, and is differentiable itself)."""

        @staticmethod
        def forward(ctx, q, k, plan, positions, back):
            ctx.plan, ctx.back = plan, back
            ctx.tensor = isinstance(positions, torch.Tensor)
            if ctx.tensor:
                ctx.save_for_backward(positions)
            else:
                ctx.positions = positions
            return _rotated(q, k, plan, positions, back)

        @staticmethod
        def backward(ctx, gq, gk):
            positions = ctx.saved_tensors[0] if ctx.tensor else ctx.positions
            gq, gk = rotary(gq, gk, ctx.plan, positions, not ctx.back)
            return gq, gk, None, None, None

    return Rotary


def rotary(q, k, plan, positions=None, back=False):
    """q and k (or None) with their positions' rotation, as new tensors; see
    kia_rotary. Differentiable."""
    import torch
    _eager(q, k)
    if torch.is_grad_enabled() and (q.requires_grad or (k is not None and k.requires_grad)):
        return _rotary_function().apply(q, k, plan, positions, back)
    return _rotated(q, k, plan, positions, back)


_rotate = rotary


# ---- attention with a sliding window ----------------------------------------------
@functools.lru_cache(maxsize=256)
def kia_window_ws_bytes(B, H, Hkv, T, d, window, sinks) -> int:
    n = ctypes.c_size_t(0)
    _kia._check(_kia.load().kia_window_ws_bytes(B, H, Hkv, T, d, window, sinks, ctypes.byref(n)))
    return n.value


def _window_checked(q, k, window, sinks, lengths):
    """(what the tensors have in common, key heads, the window, the first tokens,
    pointer of the lengths)"""
    like, Hkv = _Like("q", q), _heads(q, k)
    return like, Hkv, _int("window", window, 1), _int("sinks", sinks, 0), \
        _ints("lengths", lengths, (like.shape[0],), like.device)


def _lse(like, t):
    """Device pointer of a call's lse, contiguous [B, heads, T] (it is read and written
    flat: any other shape would be other rows)."""
    import torch
    if t.shape != like.shape[:3]:
        raise KiaError(f"lse has shape {tuple(t.shape)}, expected {tuple(like.shape[:3])}")
    return _buffer("lse", t, torch.float32, 0, like.device, 16)


def _window_fwd(c, views, lse, stream=None):
    like, Hkv, window, sinks, n = c
    B, H, T, d = like.shape
    _call(_kia.load().kia_window_fwd, like.device, stream, *views, lse, n, B, H, Hkv, T, d, window,
          sinks, like.code)


def _window_bwd(c, views, lse, ws, grads, stream=None):
    like, Hkv, window, sinks, n = c
    B, H, T, d = like.shape
    _call(_kia.load().kia_window_bwd, like.device, stream, *views, _lse(like, lse), n, ws, *grads, B, H, Hkv, T,
          d, window, sinks, like.code)


def kia_window_fwd(q, k, v, o, lse, window, sinks=0, lengths=None, stream=None):
    """Forward into o (as q) and lse ([B, H, T] float32)."""
    c = _window_checked(q, k, window, sinks, lengths)
    like, Hkv = c[:2]
    views = (like.view("q", q), like.view("k", k, Hkv), like.view("v", v, Hkv),
             like.view("o", o, out=True))
    _window_fwd(c, views, _lse(like, lse), stream)


def kia_window_bwd(q, k, v, o, dO, lse, ws, dq, dk, dv, window, sinks=0, lengths=None,
                   stream=None):
    """Backward from the forward's o and lse into dq (as q), dk and dv (as k); ws:
    a uint8 device buffer of kia_window_ws_bytes bytes, 256-byte aligned."""
    import torch
    c = _window_checked(q, k, window, sinks, lengths)
    like, Hkv, window, sinks, _ = c
    B, H, T, d = like.shape
    views = (like.view("q", q), like.view("k", k, Hkv), like.view("v", v, Hkv), like.view("o", o),
             like.view("dO", dO))
    grads = (like.view("dq", dq, out=True), like.view("dk", dk, Hkv, True),
             like.view("dv", dv, Hkv, True))
    need = kia_window_ws_bytes(B, H, Hkv, T, d, window, sinks)
    _window_bwd(c, views, lse, _buffer("ws", ws, torch.uint8, need, like.device, 256), grads, stream)


def window_forward(q, k, v, window, sinks=0, lengths=None):
    """Allocates o and lse and runs kia_window_fwd; returns (o, lse)."""
    _eager(q, k, v)
    made = _fast().window_forward(q, k, v, window, sinks, lengths)
    if made is not None:
        return made
    import torch
    c = _window_checked(q, k, window, sinks, lengths)
    like, Hkv = c[:2]
    q, vq = like.take("q", q)
    k, vk = like.take("k", k, Hkv)
    v, vv = like.take("v", v, Hkv)
    o, vo = _new(q)
    lse = torch.empty(*like.shape[:3], dtype=torch.float32, device=like.device)
    _window_fwd(c, (vq, vk, vv, vo), lse.data_ptr())
    return o, lse


def window_backward(q, k, v, o, dO, lse, window, sinks=0, lengths=None):
    """Allocates dq, dk, dv and runs kia_window_bwd; returns (dq, dk, dv)."""
    _eager(q, k, v, o, dO, lse)
    made = _fast().window_backward(q, k, v, window, sinks, lengths, o, dO, lse)
    if made is not None:
        return made
    import torch
    c = _window_checked(q, k, window, sinks, lengths)
    like, Hkv, window, sinks, _ = c
    B, H, T, d = like.shape
    q, vq = like.take("q", q)
    k, vk = like.take("k", k, Hkv)
    v, vv = like.take("v", v, Hkv)
    o, vo = like.take("o", o)
    dO, vg = like.take("dO", dO)
    (dq, gq), (dk, gk), (dv, gv) = _new(q), _new(k), _new(k)
    ws = torch.empty(kia_window_ws_bytes(B, H, Hkv, T, d, window, sinks), dtype=torch.uint8,
                     device=like.device)
    _window_bwd(c, (vq, vk, vv, vo, vg), lse, ws.data_ptr(), (gq, gk, gv))
    return dq, dk, dv


@functools.lru_cache(maxsize=1)
def _window_function():
    import torch

    class WindowAttention(torch.autograd.Function):
        """window_attention as an autograd operation; keeps o and lse for the
        backward. Not twice differentiable."""

        @staticmethod
        def forward(ctx, q, k, v, window, sinks, lengths):
            o, lse = window_forward(q, k, v, window, sinks, lengths)
            ctx.save_for_backward(q, k, v, o, lse, *([] if lengths is None else [lengths]))
            ctx.args = (window, sinks)
            return o

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dO):
            q, k, v, o, lse, *lengths = ctx.saved_tensors
            grads = window_backward(q, k, v, o, dO, lse, *ctx.args, *lengths)
            return (*grads, None, None, None)

    return WindowAttention


def window_attention(q, k, v, window, sinks=0, lengths=None, rotary=None, positions=None):
    """Differentiable causal softmax attention with a sliding window and visible
    first tokens: query i of q [B, H, T, d] sees key j of k, v [B, Hkv, T, d] iff
    j <= i and (i - j < window or j < sinks); H a multiple of Hkv. lengths:
    int32 [B], tokens of each sequence (rows past it get o = 0 and no gradient).
    rotary: a RotaryPlan that turns q and k by `positions` first."""
    import torch
    _eager(q, k, v)
    if rotary is not None:
        q, k = _rotate(q, k, rotary, positions)
    elif positions is not None:
        raise KiaError("positions without a rotary plan")
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad):
        return _window_function().apply(q, k, v, window, sinks, lengths)
    return window_forward(q, k, v, window, sinks, lengths)[0]


# ---- the 4-bit cache ---------------------------------------------------------------
PAGES = (16, 32, 64, 128, 256)


class Cache4:
    """A paged key/value cache in 4 bits: `data`, uint8 [pages, 2, heads,
    page * (d/2 + d/32)], and the head dimension (the layout is kia.h's)."""
    __slots__ = ("data", "d", "page", "pages", "heads")

    def __init__(self, data, d):
        import torch
        if d not in (32, 64, 128):
            raise KiaError(f"a 4-bit cache holds heads of 32, 64 or 128 channels, got {d!r}")
        if data.dtype != torch.uint8 or data.dim() != 4 or data.shape[1] != 2 or \
                not data.is_contiguous():
            raise KiaError("a cache's data must be contiguous uint8 [pages, 2, heads, bytes]")
        pages, _, heads, size = data.shape
        page, rest = divmod(size, d // 2 + d // 32)
        if rest or page not in PAGES or pages < 1 or heads < 1:
            raise KiaError(f"no cache of heads of {d} channels has shape {tuple(data.shape)}")
        self.data, self.d, self.page, self.pages, self.heads = data, d, page, pages, heads


def kia_cache4_bytes(pages, page, Hkv, d) -> int:
    n = ctypes.c_size_t(0)
    _kia._check(_kia.load().kia_cache4_bytes(pages, page, Hkv, d, ctypes.byref(n)))
    return n.value


def new_cache4(pages, heads, page, d, device="cuda"):
    """An empty cache (every value 0)."""
    import torch
    n = kia_cache4_bytes(_int("pages", pages, 1), page, _int("heads", heads, 1), d)
    return Cache4(torch.zeros((pages, 2, heads, n // (2 * pages * heads)), dtype=torch.uint8,
                              device=device), d)


def _cache_args(cache, table, like, heads=None):
    """(data, pages, page, table, width) after the checks that go by the cache."""
    import torch
    data = cache.data
    if data.device != like.device:
        raise KiaError(f"the cache is on {data.device}, expected {like.device}")
    ptr = data.data_ptr()
    if ptr % 16:
        raise KiaError("the cache must be 16-byte aligned")
    if like.shape[3] != cache.d:
        raise KiaError(f"the cache holds heads of {cache.d} channels, got {like.shape[3]}")
    if heads is not None and heads != cache.heads:
        raise KiaError(f"the cache holds {cache.heads} heads, got {heads}")
    if not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise KiaError("table must be an int32 tensor [B, width]")
    width = table.shape[1]
    return ptr, cache.pages, cache.page, \
        _ints("table", table, (like.shape[0], width), like.device), width


def _starts(name, starts, like):
    if starts is None:
        raise KiaError(f"{name} must be an int32 tensor")
    return _ints(name, starts, (like.shape[0],), like.device)


def _cache4_write(like, vk, vv, cache, table, starts, counts, stream=None):
    B, Hkv, T, d = like.shape
    args = _cache_args(cache, table, like, Hkv)
    _call(_kia.load().kia_cache4_write, like.device, stream, vk, vv, *args,
          _starts("starts", starts, like), _ints("counts", counts, (B,), like.device), B, Hkv, T, d,
          like.code)


def kia_cache4_write(k, v, cache, table, starts, counts=None, stream=None):
    """Writes tokens t < counts[b] (None: all) of k, v [B, heads, T, d] to positions
    starts[b] + t of the sequences whose pages table [B, width] (int32) names."""
    like = _Like("k", k)
    _cache4_write(like, like.view("k", k), like.view("v", v), cache, table, starts, counts, stream)


def _cache4_read(like, vk, vv, cache, table, starts, counts, stream=None):
    B, Hkv, T, d = like.shape
    args = _cache_args(cache, table, like, Hkv)
    _call(_kia.load().kia_cache4_read, like.device, stream, *args, _starts("starts", starts, like),
          _ints("counts", counts, (B,), like.device), vk, vv, B, Hkv, T, d, like.code)


def kia_cache4_read(cache, table, starts, k, v, counts=None, stream=None):
    """The values that the cache stands for at positions starts[b] + t into k, v
    [B, heads, T, d]; 0 where kia_cache4_write would have dropped the token."""
    like = _Like("k", k)
    _cache4_read(like, like.view("k", k, out=True), like.view("v", v, out=True), cache, table,
                 starts, counts, stream)


def cache4_write(k, v, cache, table, starts, counts=None):
    """kia_cache4_write, for tensors of any layout."""
    _eager(k, v)
    if _fast().cache4_write(k, v, cache.data, cache.page, cache.d, table, starts, counts):
        return
    like = _Like("k", k)
    k, vk = like.take("k", k)
    v, vv = like.take("v", v)
    _cache4_write(like, vk, vv, cache, table, starts, counts)


def cache4_read(cache, table, starts, T, dtype, counts=None):
    """Allocates k and v [B, heads, T, d] of `dtype` and runs kia_cache4_read."""
    import torch
    _eager()
    if not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise KiaError("table must be an int32 tensor [B, width]")
    k = torch.empty(table.shape[0], cache.heads, _int("T", T, 1), cache.d, dtype=dtype,
                    device=cache.data.device)
    made = _fast().cache4_read(k, cache.data, cache.page, cache.d, table, starts, counts)
    if made is not None:
        return made
    like = _Like("k", k)
    v, vv = _new(k)
    _cache4_read(like, View(k.data_ptr(), *_dense(k.shape)), vv, cache, table, starts, counts)
    return k, v


@functools.lru_cache(maxsize=1024)
def _cache4_ws_bytes(device, *args) -> int:
    import torch
    if device.type != "cuda":
        raise KiaError("libkia takes device tensors only")
    with torch.cuda.device(device):  # (the size goes by the device's compute units)
        return kia_cache4_ws_bytes(*args)


def kia_cache4_ws_bytes(page, width, B, H, Hkv, T, d, window=0, sinks=0) -> int:
    n = ctypes.c_size_t(0)
    _kia._check(_kia.load().kia_cache4_ws_bytes(page, width, B, H, Hkv, T, d, window, sinks,
                                                ctypes.byref(n)))
    return n.value


def _cache4_checked(q, cache, table, lengths, window, sinks):
    """(what the tensors have in common, arguments up to the lengths, bytes of workspace)"""
    like = _Like("q", q)
    B, H, T, d = like.shape
    args = _cache_args(cache, table, like)
    need = _cache4_ws_bytes(like.device, cache.page, args[4], B, H, cache.heads, T, d,
                            _int("window", window, 0), _int("sinks", sinks, 0))
    return like, (*args, _starts("lengths", lengths, like)), need


def _cache4_attn(like, args, vq, vo, ws, heads, op, window, sinks, stream=None):
    B, H, T, d = like.shape
    K, calib, tau, recon, _, _, _ = _kia._op(*op, 0, 0, 0)
    _call(_kia.load().kia_cache4_attn, like.device, stream, vq, vo, *args, ws, B, H, heads, T, d, K,
          calib, tau, recon, window, sinks, like.code)


def kia_cache4_attn(q, o, cache, table, lengths, ws, K=4, calib="fwm", tau=8.0, recon="nearest",
                    window=0, sinks=0, stream=None):
    """Attention of the last T tokens of each sequence, q [B, H, T, d], over its
    lengths[b] keys (the new tokens' own among them) into o; ws: a uint8 device
    buffer of kia_cache4_ws_bytes bytes, 256-byte aligned."""
    import torch
    like, args, need = _cache4_checked(q, cache, table, lengths, window, sinks)
    _cache4_attn(like, args, like.view("q", q), like.view("o", o, out=True),
                 _buffer("ws", ws, torch.uint8, need, like.device, 256), cache.heads,
                 (K, calib, tau, recon), window, sinks, stream)


def cache4_attention(q, cache, table, lengths, K=4, calib="fwm", tau=8.0, recon="nearest",
                     window=0, sinks=0, pages=None, shared=0):
    """Allocates the output (as q) and the workspace and runs kia_cache4_attn; the
    operator's arguments are those of k_interval_attention. Forward only.
    pages: only over these pages of each token and key head (cache4_select's, or any
    int32 [B, heads, T, count] of their numbers in the table). shared: the first tokens
    that all sequences have on the same pages, computed once for all."""
    import torch
    if q.requires_grad and torch.is_grad_enabled():
        raise KiaError("attention over a 4-bit cache is forward only: call it under torch.no_grad")
    _eager(q)
    op = _kia._op(K, calib, tau, recon, 0, 0, 0)
    if pages is not None or shared:
        return _served(q, cache, table, lengths, op, window, sinks, pages, shared)
    made = _fast().cache4_attention(q, cache.data, cache.page, cache.d, table, lengths, *op[:4],
                                    window, sinks)
    if made is not None:
        return made
    like, args, need = _cache4_checked(q, cache, table, lengths, window, sinks)
    q, vq = like.take("q", q)
    o, vo = _new(q)
    ws = torch.empty(need, dtype=torch.uint8, device=like.device)
    _cache4_attn(like, args, vq, vo, ws.data_ptr(), cache.heads,
                 (K, calib, tau, recon), window, sinks)
    return o


# ---- many and long texts from the cache ----------------------------------------------
def _bytes(name):
    """The binding of a workspace size."""
    def call(*args) -> int:
        n = ctypes.c_size_t(0)
        _kia._check(getattr(_kia.load(), name)(*args, ctypes.byref(n)))
        return n.value
    call.__name__ = name
    return call


kia_cache4_select_ws_bytes = _bytes("kia_cache4_select_ws_bytes")
kia_cache4_pages_ws_bytes = _bytes("kia_cache4_pages_ws_bytes")
kia_cache4_shared_ws_bytes = _bytes("kia_cache4_shared_ws_bytes")


@functools.lru_cache(maxsize=1024)
def _ws_on(device, size, *args) -> int:
    import torch
    if device.type != "cuda":
        raise KiaError("libkia takes device tensors only")
    with torch.cuda.device(device):  # (the size goes by the device's compute units)
        return size(*args)


def new_bounds4(cache):
    """Bounds of a cache's pages, to be filled: bfloat16 [pages, heads, 2, d] (the least
    and the largest key of each channel)."""
    import torch
    return torch.zeros((cache.pages, cache.heads, 2, cache.d), dtype=torch.bfloat16,
                       device=cache.data.device)


def _bounds(cache, bounds):
    import torch
    if not isinstance(bounds, torch.Tensor) or bounds.dtype != torch.bfloat16 or \
            bounds.shape != (cache.pages, cache.heads, 2, cache.d):
        raise KiaError(f"bounds must be a bfloat16 tensor [{cache.pages}, {cache.heads}, 2, {cache.d}]")
    return _buffer("bounds", bounds, torch.bfloat16, 1, cache.data.device, 16)


def _append(like, views, cache, table, starts, plan, counts, bounds, H, stream=None):
    import torch
    B, Hkv, T, d = like.shape
    ptr, *rest = _cache_args(cache, table, like, Hkv)
    freq = plan.freq
    if freq.dim() != 1 or not 2 <= 2 * freq.shape[0] <= d:
        raise KiaError(f"a plan's frequencies must be one to {d // 2} in one dimension for heads of "
                       f"{d} channels, got shape {tuple(freq.shape)}")
    if plan.layout not in LAYOUT:
        raise KiaError(f"layout must be one of {sorted(LAYOUT)}, got {plan.layout!r}")
    _call(_kia.load().kia_cache4_append, like.device, stream, *views, ptr,
          None if bounds is None else _bounds(cache, bounds), *rest, _starts("starts", starts, like),
          _ints("counts", counts, (B,), like.device),
          _buffer("the plan's frequencies", freq, torch.float64, 1, like.device, 8), float(plan.factor),
          LAYOUT[plan.layout], B, H, Hkv, T, d, 2 * freq.shape[0], like.code)


def kia_cache4_append(q, q_out, k, v, cache, table, starts, plan, counts=None, bounds=None, stream=None):
    """Appends tokens t < counts[b] (None: all) of k, v [B, heads, T, d] at positions
    starts[b] + t of the sequences whose pages table [B, width] (int32) names, k turned
    by its position, and q [B, H, T, d] turned into q_out. bounds (new_bounds4): those of
    the pages that tokens went to are brought up to date."""
    like, H = _Like("k", k), _heads(k, q)
    _append(like, (like.view("q", q, H), like.view("q_out", q_out, H, True), like.view("k", k),
                   like.view("v", v)), cache, table, starts, plan, counts, bounds, H, stream)


def cache4_append(q, k, v, cache, table, starts, plan, counts=None, bounds=None):
    """kia_cache4_append, for tensors of any layout; returns the turned q. Forward only."""
    import torch
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad):
        raise KiaError("appending to a 4-bit cache is forward only: call it under torch.no_grad")
    _eager(q, k, v)
    made = _fast().cache4_append(q, k, v, cache.data, cache.page, cache.d, table, starts, counts, plan.freq,
                                 plan.factor, LAYOUT.get(plan.layout, -1), bounds)
    if made is not None:
        return made
    like, H = _Like("k", k), _heads(k, q)
    q, vq = like.take("q", q, H)
    k, vk = like.take("k", k)
    v, vv = like.take("v", v)
    out, vo = _new(q)
    _append(like, (vq, vo, vk, vv), cache, table, starts, plan, counts, bounds, H)
    return out


def kia_cache4_bounds(cache, bounds, table, starts, ends, stream=None):
    """Brings the bounds of the pages that hold positions starts[b] .. ends[b] - 1 up to
    date, over their tokens before ends[b] (for tokens that kia_cache4_write held)."""
    device = cache.data.device
    if table.dim() != 2:
        raise KiaError("table must be an int32 tensor [B, width]")
    B, width = table.shape
    if starts is None or ends is None:
        raise KiaError("starts and ends must be int32 tensors")
    if cache.data.data_ptr() % 16:
        raise KiaError("the cache must be 16-byte aligned")
    _call(_kia.load().kia_cache4_bounds, device, stream, cache.data.data_ptr(), _bounds(cache, bounds),
          cache.pages, cache.page, _ints("table", table, (B, width), device), width,
          _ints("starts", starts, (B,), device), _ints("ends", ends, (B,), device), B, cache.heads, cache.d)


def cache4_bounds(cache, bounds, table, starts, ends):
    """kia_cache4_bounds, on the current stream."""
    _eager()
    kia_cache4_bounds(cache, bounds, table, starts, ends)


def _select(like, vq, cache, bounds, table, lengths, ws, pages, count, first, last, stream=None):
    B, H, T, d = like.shape
    _, *rest = _cache_args(cache, table, like)
    if pages.shape != (B, cache.heads, T, count):
        raise KiaError(f"pages has shape {tuple(pages.shape)}, expected {(B, cache.heads, T, count)}")
    _call(_kia.load().kia_cache4_select, like.device, stream, vq, _bounds(cache, bounds), *rest,
          _starts("lengths", lengths, like), ws, _ints("pages", pages, pages.shape, like.device), count,
          first, last, B, H, cache.heads, T, d, like.code)


def _select_checked(q, cache, table, count, first, last):
    _int("count", count, 1), _int("first", first, 0), _int("last", last, 1)
    if first + last > count:
        raise KiaError(f"count must be at least first + last, got {count}")
    like = _Like("q", q)
    B, H, T, d = like.shape
    width = _cache_args(cache, table, like)[4]
    return like, _ws_on(like.device, kia_cache4_select_ws_bytes, cache.page, width, B, H, cache.heads, T, d)


def kia_cache4_select(q, pages, cache, bounds, table, lengths, ws, first=1, last=1, stream=None):
    """The pages that each of the last T tokens, q [B, H, T, d], reads of its sequence's
    lengths[b] keys, into pages (int32 [B, heads, T, count]); ws: a uint8 device buffer of
    kia_cache4_select_ws_bytes bytes, 256-byte aligned."""
    import torch
    if pages.dim() != 4:
        raise KiaError(f"pages must be [B, heads, T, count], got shape {tuple(pages.shape)}")
    count = pages.shape[3]
    like, need = _select_checked(q, cache, table, count, first, last)
    _select(like, like.view("q", q), cache, bounds, table, lengths,
            _buffer("ws", ws, torch.uint8, need, like.device, 256), pages, count, first, last, stream)


def cache4_select(q, cache, bounds, table, lengths, count, first=1, last=1):
    """Allocates and returns the pages that kia_cache4_select takes: for each token and
    key head `count` numbers of pages in the table, ascending, -1 behind them; the first and
    the last ones and those whose bounds allow the highest score with any of the key
    head's queries. For cache4_attention(..., pages=)."""
    import torch
    _eager(q)
    made = _fast().cache4_select(q, cache.data, cache.page, cache.d, table, lengths, bounds, count, first, last)
    if made is not None:
        return made
    like, need = _select_checked(q, cache, table, count, first, last)
    q, vq = like.take("q", q)
    B, H, T, d = like.shape
    pages = torch.empty((B, cache.heads, T, count), dtype=torch.int32, device=like.device)
    ws = torch.empty(need, dtype=torch.uint8, device=like.device)
    _select(like, vq, cache, bounds, table, lengths, ws.data_ptr(), pages, count, first, last)
    return pages


def _pages_checked(q, cache, table, lengths, pages):
    """(what the tensors have in common, arguments up to the workspace, its bytes)"""
    import torch
    if not isinstance(pages, torch.Tensor) or pages.dim() != 4:
        raise KiaError("pages must be an int32 tensor [B, heads, T, count]")
    like = _Like("q", q)
    B, H, T, d = like.shape
    args, count = _cache_args(cache, table, like), pages.shape[3]
    n, ptr = _starts("lengths", lengths, like), _ints("pages", pages, (B, cache.heads, T, count), like.device)
    need = _ws_on(like.device, kia_cache4_pages_ws_bytes, cache.page, args[4], count, B, H, cache.heads, T, d)
    return like, (*args, n, ptr, count), need


def _shared_checked(q, cache, table, lengths, shared):
    like = _Like("q", q)
    B, H, T, d = like.shape
    args = _cache_args(cache, table, like)
    if _int("shared", shared, 1) % max(32, cache.page):
        raise KiaError(f"shared must be a multiple of {max(32, cache.page)} tokens, got {shared}")
    if shared > args[4] * cache.page:
        raise KiaError(f"shared passes the table's {args[4] * cache.page} tokens, got {shared}")
    need = _ws_on(like.device, kia_cache4_shared_ws_bytes, cache.page, args[4], shared, B, H, cache.heads, T, d)
    return like, (*args, _starts("lengths", lengths, like), shared), need


def _served_call(name, like, args, vq, vo, ws, heads, op, stream=None):
    B, H, T, d = like.shape
    K, calib, tau, recon = op[:4]
    _call(getattr(_kia.load(), name), like.device, stream, vq, vo, *args, ws, B, H, heads, T, d, K, calib,
          tau, recon, like.code)


def kia_cache4_attn_pages(q, o, cache, table, lengths, pages, ws, K=4, calib="fwm", tau=8.0, recon="nearest",
                          stream=None):
    """kia_cache4_attn of which token t and key head h see only the pages that
    pages[b, h, t] names; ws: kia_cache4_pages_ws_bytes bytes."""
    import torch
    like, args, need = _pages_checked(q, cache, table, lengths, pages)
    _served_call("kia_cache4_attn_pages", like, args, like.view("q", q), like.view("o", o, out=True),
                 _buffer("ws", ws, torch.uint8, need, like.device, 256), cache.heads,
                 _kia._op(K, calib, tau, recon, 0, 0, 0), stream)


def kia_cache4_attn_shared(q, o, cache, table, lengths, shared, ws, K=4, calib="fwm", tau=8.0, recon="nearest",
                           stream=None):
    """kia_cache4_attn for sequences whose first `shared` tokens are on the same pages
    (those of the table's first row); ws: kia_cache4_shared_ws_bytes bytes."""
    import torch
    like, args, need = _shared_checked(q, cache, table, lengths, shared)
    _served_call("kia_cache4_attn_shared", like, args, like.view("q", q), like.view("o", o, out=True),
                 _buffer("ws", ws, torch.uint8, need, like.device, 256), cache.heads,
                 _kia._op(K, calib, tau, recon, 0, 0, 0), stream)


def _served(q, cache, table, lengths, op, window, sinks, pages, shared):
    """cache4_attention over listed pages or behind shared tokens."""
    import torch
    if pages is not None and shared:
        raise KiaError("pages and shared tokens are not taken together")
    if window != 0 or sinks != 0:
        raise KiaError("a window is not taken with pages or shared tokens")
    made = _fast().cache4_served(q, cache.data, cache.page, cache.d, table, lengths, pages, shared, *op[:4])
    if made is not None:
        return made
    if pages is not None:
        name, (like, args, need) = "kia_cache4_attn_pages", _pages_checked(q, cache, table, lengths, pages)
    else:
        name, (like, args, need) = "kia_cache4_attn_shared", _shared_checked(q, cache, table, lengths, shared)
    q, vq = like.take("q", q)
    o, vo = _new(q)
    ws = torch.empty(need, dtype=torch.uint8, device=like.device)
    _served_call(name, like, args, vq, vo, ws.data_ptr(), cache.heads, op)
    return o
