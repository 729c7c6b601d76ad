"""Rotary positions: binding of include/uzip_rotary.h.

``rotate`` turns queries or keys (and, with ``inverse``, gradients: it is
differentiable itself), ``kv_rotate_store`` turns keys on their way into a
``KVCache`` and the step's queries beside them, ``kv_positions`` gives the places
that both go by from what ``kv_plan`` leaves.  ``rotary_frequencies`` makes the
frequencies, also scaled for contexts longer than a model was trained on.
"""
from __future__ import annotations

import ctypes
import math

import torch
import torch.autograd.forward_ad as _forward

from . import OK, _check, _lib
from .kv import KVCache, _TYPES, _cache_p, _current, _device, _handle, _i64, _int, _ints, _on, _rows, _u32, _vp, _apart, _wrote

_c = ctypes


class uzip_turn(_c.Structure):
    _fields_ = [("positions", _vp), ("freq", _vp), ("rot", _u32), ("first", _u32), ("interleaved", _u32), ("inverse", _u32),
                ("magnitude", _c.c_double)]


_turn_p = _c.POINTER(uzip_turn)
_lib.uzip_kv_positions.argtypes = [_vp, _vp, _u32, _u32, _vp, _vp]
_lib.uzip_kv_positions.restype = _int
_lib.uzip_rotate.argtypes = [_int, _vp, _i64, _i64, _u32, _u32, _u32, _turn_p, _vp, _i64, _i64, _vp]
_lib.uzip_rotate.restype = _int
_lib.uzip_kv_rotate_store.argtypes = [_cache_p, _int, _vp, _i64, _i64, _vp, _i64, _i64, _u32, _vp, _vp, _vp, _u32, _turn_p, _vp, _i64,
                                      _i64, _u32, _vp, _i64, _i64, _vp]
_lib.uzip_kv_rotate_store.restype = _int

EXPORTED = ["uzip_kv_positions", "uzip_rotate", "uzip_kv_rotate_store"]

uzip_kv_positions = _lib.uzip_kv_positions
uzip_rotate = _lib.uzip_rotate
uzip_kv_rotate_store = _lib.uzip_kv_rotate_store


def rotary_frequencies(rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, trained: int = 0,
                       fast: float = 32.0, slow: float = 1.0, device="cuda"):
    """(frequencies fp32 [rot / 2], magnitude) of a rotary part of ``rot`` channels: base^(-2 i / rot) radians a position.

    ``scaling`` for contexts ``factor`` times as long as the ``trained`` one:
    "linear": positions are divided by the factor; "base": the base is raised so that
    the slowest pair is, and the fastest stays (base * factor^(rot / (rot - 2)));
    "parts": pairs that turn more than ``fast`` times over the trained length stay,
    those that turn less than ``slow`` times are divided, the ones between go
    linearly from one to the other by their number, and the magnitude is
    0.1 ln(factor) + 1 (arXiv 2309.00071)."""
    if rot < 2 or rot % 2 or not base > 1 or not factor >= 1 or scaling not in ("none", "linear", "base", "parts"):
        raise ValueError("rot is even, base above 1, factor at least 1, scaling one of none, linear, base, parts")
    magnitude = 1.0
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    i = torch.arange(rot // 2, dtype=torch.float64)
    freq = base ** (-2.0 * i / rot)
    if scaling == "linear":
        freq = freq / factor
    elif scaling == "parts":
        if trained < 1 or not fast > slow > 0:
            raise ValueError("scaling by parts needs the trained length, and fast above slow")

        def number(turns):                                      # of the pair that turns so often over the trained length
            return rot * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base))
        low, high = max(math.floor(number(fast)), 0), min(math.ceil(number(slow)), rot - 1)   # may lie past the last pair
        divided = ((i - low) / max(high - low, 1e-3)).clamp(0, 1)
        freq = freq * (1 - divided) + freq / factor * divided
        magnitude = 0.1 * math.log(factor) + 1
    return freq.float().to(device), magnitude


def _turn(positions: torch.Tensor, freq: torch.Tensor, rows: int, device: int, interleaved: bool, first: int, magnitude: float,
          inverse: bool) -> uzip_turn:
    _ints(positions, "positions", device)
    if freq.get_device() != device or freq.dtype is not torch.float32 or freq.dim() != 1 or not freq.is_contiguous():
        raise ValueError("freq is a contiguous fp32 vector on the current GPU")
    if positions.numel() < rows:
        raise ValueError("positions has an entry for each row")
    half = freq.numel()
    if not 0 <= first <= 1024 or not 1 <= half <= 512:
        raise ValueError("the rotary part is 2 to 1024 channels from first on")
    return uzip_turn(positions.data_ptr(), freq.data_ptr(), 2 * half, first, bool(interleaved), bool(inverse), magnitude)


def kv_positions(lens: torch.Tensor, q_start: torch.Tensor, rows: int, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """int32 [rows]: each new token's place in its request, from ``lens`` and ``q_start`` as kv_plan leaves them; -1 for
    rows of no request."""
    device = _device()
    _ints(lens, "lens", device)
    _ints(q_start, "q_start", device)
    if q_start.numel() <= lens.numel():
        raise ValueError("lens and q_start are of one batch")
    if not 0 <= rows < 1 << 31:
        raise ValueError("rows is not negative")
    given = out
    if out is None:
        with _on(stream):
            out = torch.empty(rows, dtype=torch.int32, device=lens.device)
    _ints(out, "out", device)
    if out.numel() < rows:
        raise ValueError("out has an entry for each row")
    rc = uzip_kv_positions(lens.data_ptr(), q_start.data_ptr(), lens.numel(), rows, out.data_ptr(), _handle(stream, device))
    if rc != OK:
        _check(rc, "uzip_kv_positions")
    _wrote(given)
    return out


def _rotate(x, positions, freq, interleaved, first, magnitude, inverse, out, stream):
    device = _device()
    if x.dim() != 3:
        raise ValueError("x is [rows, heads, dim]")
    t = _rows(x, "x", x.shape[2], device)
    rows, heads, dim = x.shape
    turn = _turn(positions, freq, rows, device, interleaved, first, magnitude, inverse)
    if first + turn.rot > dim:
        raise ValueError("the rotary part lies within dim")
    given = out
    _apart(out, "out")
    if out is None:
        with _on(stream):
            out = torch.empty(rows, heads, dim, dtype=x.dtype, device=x.device)
    if _rows(out, "out", dim, device) != t or out.shape != x.shape:
        raise ValueError("out is like x")
    rc = uzip_rotate(t, x.data_ptr(), x.stride(0), x.stride(1), rows, heads, dim, _c.byref(turn), out.data_ptr(), out.stride(0),
                     out.stride(1), _handle(stream, device))
    if rc != OK:
        _check(rc, "uzip_rotate")
    _wrote(given)
    return out


def _followed(x) -> bool:
    """Whether autograd follows x, backwards or forwards."""
    return (x.requires_grad and torch.is_grad_enabled()) or (_forward._current_level >= 0 and _forward.unpack_dual(x).tangent is not None)


class _Rotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, positions, freq, interleaved, first, magnitude, inverse):
        ctx.save_for_backward(positions, freq)
        ctx.save_for_forward(positions, freq)
        ctx.how = interleaved, first, magnitude, inverse
        return _rotate(x, positions, freq, interleaved, first, magnitude, inverse, None, None)

    @staticmethod
    def backward(ctx, grad):
        positions, freq = ctx.saved_tensors
        interleaved, first, magnitude, inverse = ctx.how
        if grad.stride(2) != 1:
            grad = grad.contiguous()
        # through apply, so that a gradient of the gradient is had the same way
        return _Rotate.apply(grad, positions, freq, interleaved, first, magnitude, not inverse), None, None, None, None, None, None

    @staticmethod
    def jvp(ctx, tangent, *_):
        positions, freq = ctx.saved_tensors
        if tangent.stride(2) != 1:
            tangent = tangent.contiguous()
        return _Rotate.apply(tangent, positions, freq, *ctx.how)          # linear in x


def rotate(x: torch.Tensor, positions: torch.Tensor, freq: torch.Tensor, interleaved: bool = False, first: int = 0,
           magnitude: float = 1.0, inverse: bool = False, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """x [rows, heads, dim] with channels first .. first + 2 freq.numel() turned by positions[row] * freq: pairs
    (i, i + rot / 2), or (2 i, 2 i + 1) where ``interleaved``, times ``magnitude``; by the angles' negatives with
    ``inverse``.  ``out`` may be x.  Differentiable in x where neither out nor stream is given, and not in freq."""
    if _followed(freq):
        raise ValueError("no gradient goes to the frequencies: detach them")
    if _followed(x) or (out is not None and _followed(out)):
        if out is not None or stream is not None:
            raise ValueError("a rotation that is differentiated takes neither out nor stream")
        return _Rotate.apply(x, positions, freq, interleaved, first, magnitude, inverse)
    return _rotate(x, positions, freq, interleaved, first, magnitude, inverse, out, stream)


def _serves(*tensors) -> None:
    for x in tensors:
        if x is not None and _followed(x):
            raise ValueError("no gradient goes through this call: detach its inputs, or call it under torch.no_grad()")


def _queries(q, q_out, rows: int, dim: int, device: int, kind: int, stream):
    """(x, out) of the queries that are turned beside a store, or (None, None)."""
    if q is None:
        if q_out is not None:
            raise ValueError("q_out is for q")
        return None, None
    if _rows(q, "q", dim, device) != kind or q.shape[0] != rows:
        raise ValueError("q has the rows and the type of what is stored")
    _apart(q_out, "q_out")
    if q_out is None:
        with _on(stream):
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if _rows(q_out, "q_out", dim, device) != kind or q_out.shape != q.shape:
        raise ValueError("q_out is like q")
    return q, q_out


def _query_args(q, q_out):
    if q is None:
        return None, 0, 0, 0, None, 0, 0
    step, out_step = q.stride(), q_out.stride()
    return q.data_ptr(), step[0], step[1], q.shape[1], q_out.data_ptr(), out_step[0], out_step[1]


def kv_rotate_store(cache: KVCache, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, freq: torch.Tensor, slots: torch.Tensor,
                    runs: torch.Tensor, counts: torch.Tensor, q: torch.Tensor | None = None, interleaved: bool = False, first: int = 0,
                    magnitude: float = 1.0, q_out: torch.Tensor | None = None, stream=None):
    """kv_store with the keys turned on the way (their codes are the only rounding), and the step's queries
    q [rows, query heads, dim] turned in the same launch.  No gradient goes through it.  Returns q_out, None without q."""
    device = _current(cache)
    _serves(k, v, q, q_out, freq)
    t = _rows(k, "k", cache.dim, device)
    shape = k.shape
    if _rows(v, "v", cache.dim, device) != t or v.shape != shape or shape[1] != cache.heads:
        raise ValueError("k and v are [rows, the cache's heads, dim] of one type")
    _ints(slots, "slots", device, torch.int64)
    _ints(runs, "runs", device)
    _ints(counts, "counts", device)
    rows, n_runs = shape[0], runs.shape[0]
    if slots.numel() < rows or counts.numel() < 2 or runs.numel() != 2 * n_runs:
        raise ValueError("slots has an entry for each row, runs two for each run, counts two")
    turn = _turn(positions, freq, rows, device, interleaved, first, magnitude, False)
    if first + turn.rot > cache.dim:
        raise ValueError("the rotary part lies within dim")
    given = q_out
    q, q_out = _queries(q, q_out, rows, cache.dim, device, t, stream)
    k_step, v_step = k.stride(), v.stride()
    rc = uzip_kv_rotate_store(cache, t, k.data_ptr(), k_step[0], k_step[1], v.data_ptr(), v_step[0], v_step[1], rows,
                              slots.data_ptr(), runs.data_ptr(), counts.data_ptr(), n_runs, _c.byref(turn), *_query_args(q, q_out),
                              _handle(stream, device))
    if rc != OK:
        _check(rc, "uzip_kv_rotate_store")
    _wrote(given)
    return q_out
