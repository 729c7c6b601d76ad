"""Latent attention: binding of include/uzip_latent.h.

``LatentCache`` holds a pool of pages with one latent vector and one rotary key a
token in 8 bits; ``latent_store`` writes new tokens, ``latent_attend`` lets them
attend to their requests' pages (absorbed form), ``latent_attend_expanded`` is
attention over a prompt's keys and values made from the latents (expanded form).
Places come from ``kv_plan`` and ``kv_positions``.  These calls serve: no gradient
goes through them.
"""
from __future__ import annotations

import ctypes

import torch

from . import BF16, EINVAL, FP16, OK, _check, _dev_empty, _lib
from .kv import _CODES, _TYPES, _device, _handle, _i64, _int, _ints, _need, _on, _rows, _sz, _u32, _vp, _f32, _apart, _wrote
from .rotary import _queries, _query_args, _serves, _turn, _turn_p

_c = ctypes


class uzip_latent_cache(_c.Structure):
    _fields_ = [("codes", _vp), ("exps", _vp), ("n_pages", _u32), ("latent", _u32), ("rot", _u32), ("page_tokens", _u32), ("dtype", _int)]


_latent_p = _c.POINTER(uzip_latent_cache)
_lib.uzip_latent_store.argtypes = [_latent_p, _int, _vp, _i64, _vp, _i64, _u32, _vp, _turn_p, _vp, _i64, _i64, _u32, _vp, _i64, _i64, _vp]
_lib.uzip_latent_store.restype = _int
_lib.uzip_latent_attend_workspace.argtypes = [_u32, _u32, _u32, _u32, _u32]
_lib.uzip_latent_attend_workspace.restype = _sz
_lib.uzip_latent_attend.argtypes = [_latent_p, _int, _vp, _i64, _i64, _u32, _u32, _vp, _u32, _vp, _vp, _u32, _u32, _f32, _vp, _i64, _i64,
                                    _vp, _vp, _sz, _vp]
_lib.uzip_latent_attend.restype = _int
_lib.uzip_latent_attend_expanded.argtypes = [_int, _vp, _i64, _i64, _u32, _u32, _vp, _i64, _i64, _vp, _i64, _vp, _i64, _i64, _u32, _u32, _u32,
                                             _u32, _vp, _vp, _u32, _u32, _f32, _vp, _i64, _i64, _vp, _vp]
_lib.uzip_latent_attend_expanded.restype = _int

EXPORTED = ["uzip_latent_store", "uzip_latent_attend_workspace", "uzip_latent_attend",
            "uzip_latent_attend_expanded"]

uzip_latent_store = _lib.uzip_latent_store
uzip_latent_attend_workspace = _lib.uzip_latent_attend_workspace
uzip_latent_attend = _lib.uzip_latent_attend
uzip_latent_attend_expanded = _lib.uzip_latent_attend_expanded


class LatentCache:
    """Pages of latents and rotary keys in 8 bits.

    codes [pages, page tokens, latent + rot], uint8 codes of ``dtype`` ("e4m3fn" or
    "e5m2"), a token's latent before its rotary key; exps [pages, page tokens, 2], uint8: a
    value is code * 2^(exponent - 127), the first exponent for the latent.
    """

    def __init__(self, codes: torch.Tensor, exps: torch.Tensor, rot: int, dtype="e4m3fn"):
        _need(codes.dim() == 3 and 0 < rot < codes.shape[2], "codes is [pages, page tokens, latent + rot]")
        pages, page, width = codes.shape
        _need(tuple(exps.shape) == (pages, page, 2), "exps is [pages, page tokens, 2]")
        for x in (codes, exps):
            _need(x.is_cuda and x.device == codes.device and x.is_contiguous() and x.element_size() == 1,
                  "the cache's arrays are contiguous bytes on one GPU")
        _need(dtype in _CODES, "dtype is e4m3fn or e5m2")
        self.codes, self.exps = codes, exps
        self.pages, self.page_tokens, self.latent, self.rot = pages, page, width - rot, rot
        self.code, self.device, self.index = _CODES[dtype], codes.device, codes.get_device()
        self.desc = uzip_latent_cache(codes.data_ptr(), exps.data_ptr(), pages, self.latent, rot, page, self.code)
        self._as_parameter_ = _c.byref(self.desc)

    @classmethod
    def empty(cls, pages: int, latent: int = 512, rot: int = 64, page_tokens: int = 64, dtype="e4m3fn", device="cuda") -> "LatentCache":
        """A pool of unwritten pages."""
        def new(*shape):
            return torch.empty(*shape, dtype=torch.uint8, device=device)
        return cls(new(pages, page_tokens, latent + rot), new(pages, page_tokens, 2), rot, dtype)


def _current(cache: LatentCache) -> int:
    device = _device()
    if cache.index != device:
        raise ValueError("the cache is on another GPU than the current one")
    return device


def _vectors(x: torch.Tensor, name: str, dim: int, device: int) -> int:
    t = _TYPES.get(x.dtype)
    if t is None or x.get_device() != device or x.dim() != 2 or x.shape[1] != dim or (x.stride(1) != 1 and x.numel()):
        raise ValueError(f"{name} is [rows, {dim}] in bf16, fp16 or fp32 on the current GPU with each row's values side by side")
    return t


def latent_store(cache: LatentCache, latent: torch.Tensor, key_rot: torch.Tensor, positions: torch.Tensor, freq: torch.Tensor,
                 slots: torch.Tensor, q: torch.Tensor | None = None, interleaved: bool = False, magnitude: float = 1.0,
                 q_out: torch.Tensor | None = None, stream=None):
    """Write rows of latents [rows, latent] and rotary keys [rows, rot], turned on the way, to the slots that kv_plan
    made (no slot twice); the queries' rotary parts q [rows, heads, rot] are turned into q_out in the same launch.
    Returns q_out, None without q."""
    device = _current(cache)
    _serves(latent, key_rot, q, q_out, freq)
    t = _vectors(latent, "latent", cache.latent, device)
    rows = latent.shape[0]
    if _vectors(key_rot, "key_rot", cache.rot, device) != t or key_rot.shape[0] != rows:
        raise ValueError("latent and key_rot are of one type and as many rows")
    _ints(slots, "slots", device, torch.int64)
    if slots.numel() < rows:
        raise ValueError("slots has an entry for each row")
    turn = _turn(positions, freq, rows, device, interleaved, 0, magnitude, False)
    if turn.rot != cache.rot:
        raise ValueError("freq is for the cache's rotary keys")
    given = q_out
    q, q_out = _queries(q, q_out, rows, cache.rot, device, t, stream)
    rc = uzip_latent_store(cache, t, latent.data_ptr(), latent.stride(0), key_rot.data_ptr(), key_rot.stride(0), rows, slots.data_ptr(),
                           _c.byref(turn), *_query_args(q, q_out), _handle(stream, device))
    if rc != OK:
        _check(rc, "uzip_latent_store")
    _wrote(given)
    return q_out


def _attend_type(t: int, what: str) -> int:
    if t not in (BF16, FP16):
        raise ValueError(f"{what} is bf16 or fp16")
    return t


def latent_attend_workspace(q: torch.Tensor, cache: LatentCache, requests: int, max_new: int) -> torch.Tensor:
    _attend_type(_rows(q, "q", cache.latent + cache.rot, cache.index), "q")
    if not (0 <= requests < 1 << 32 and 0 <= max_new < 1 << 32):
        raise ValueError("requests and max_new are not negative")
    n = uzip_latent_attend_workspace(cache.latent, q.shape[0], q.shape[1], requests, max_new)
    if n == 0:
        _check(EINVAL, "uzip_latent_attend_workspace")
    return _dev_empty(n, q.device)


def latent_attend(q: torch.Tensor, cache: LatentCache, table: torch.Tensor, lens: torch.Tensor, q_start: torch.Tensor, max_new: int,
                  scale: float, out: torch.Tensor | None = None, lse: torch.Tensor | None = None, ws: torch.Tensor | None = None,
                  stream=None):
    """Causal attention of the new tokens q [rows, heads, latent + rot] over their requests' pages, every head over the
    same latents.  ``scale`` is that of the expanded form's keys.  Returns (out [rows, heads, latent], lse [rows, heads] fp32)."""
    device = _current(cache)
    _serves(q, out, lse)
    t = _attend_type(_rows(q, "q", cache.latent + cache.rot, device), "q")
    rows, heads = q.shape[0], q.shape[1]
    n = lens.numel()
    _ints(table, "table", device)
    _ints(lens, "lens", device)
    _ints(q_start, "q_start", device)
    if table.dim() != 2 or table.shape[0] < n or q_start.numel() <= n:
        raise ValueError("table, lens and q_start are of one batch")
    if not 0 <= max_new < 1 << 32:
        raise ValueError("max_new is not negative")
    given = out, lse
    _apart(out, "out")
    if out is None or lse is None or ws is None:
        with _on(stream):
            out = torch.empty(rows, heads, cache.latent, dtype=q.dtype, device=q.device) if out is None else out
            lse = torch.empty(rows, heads, dtype=torch.float32, device=q.device) if lse is None else lse
            ws = latent_attend_workspace(q, cache, n, max_new) if ws is None else ws
    if _rows(out, "out", cache.latent, device) != t or out.shape[:2] != q.shape[:2]:
        raise ValueError("out is [rows, heads, latent] of q's type")
    if lse.get_device() != device or lse.dtype != torch.float32 or not lse.is_contiguous() or lse.shape != q.shape[:2]:
        raise ValueError("lse is fp32 [rows, heads]")
    if ws.get_device() != device or not ws.is_contiguous():
        raise ValueError("ws is a contiguous tensor on the current GPU")
    rc = uzip_latent_attend(cache, t, q.data_ptr(), q.stride(0), q.stride(1), rows, heads, table.data_ptr(), table.shape[1], lens.data_ptr(),
                            q_start.data_ptr(), n, max_new, scale, out.data_ptr(), out.stride(0), out.stride(1), lse.data_ptr(),
                            ws.data_ptr(), ws.numel() * ws.element_size(), _handle(stream, device))
    if rc != OK:
        _check(rc, "uzip_latent_attend")
    _wrote(*given)
    return out, lse


def latent_attend_expanded(q: torch.Tensor, k: torch.Tensor, key_rot: torch.Tensor, v: torch.Tensor, q_start: torch.Tensor,
                           k_start: torch.Tensor, max_new: int, scale: float | None = None, out: torch.Tensor | None = None,
                           lse: torch.Tensor | None = None, stream=None):
    """Causal attention of prompts in the expanded form: q [rows, heads, nope + rot], k [keys, heads, nope], key_rot
    [keys, rot] (turned already, the same for all heads), v [keys, heads, value].  Request i has the rows from q_start[i]
    and the keys from k_start[i] on, up to the next request's; its last row sees all of its keys.  Returns (out [rows,
    heads, value], lse [rows, heads] fp32)."""
    device = _device()
    _serves(q, k, key_rot, v, out, lse)
    if q.dim() != 3 or k.dim() != 3 or key_rot.dim() != 2 or v.dim() != 3:
        raise ValueError("q, k and v are [rows or keys, heads, dim], key_rot is [keys, rot]")
    nope, rot, value = k.shape[2], key_rot.shape[1], v.shape[2]
    t = _attend_type(_rows(q, "q", nope + rot, device), "q")
    rows, heads, keys = q.shape[0], q.shape[1], k.shape[0]
    if (_rows(k, "k", nope, device) != t or _vectors(key_rot, "key_rot", rot, device) != t or _rows(v, "v", value, device) != t
            or key_rot.shape[0] != keys or v.shape[0] != keys or k.shape[1] != heads or v.shape[1] != heads):
        raise ValueError("k, key_rot and v have as many keys, the queries' heads and their type")
    _ints(q_start, "q_start", device)
    _ints(k_start, "k_start", device)
    n = k_start.numel() - 1
    if n < 0 or q_start.numel() <= n:
        raise ValueError("q_start and k_start are of one batch")
    if not 0 <= max_new < 1 << 32:
        raise ValueError("max_new is not negative")
    given = out, lse
    _apart(out, "out")
    if out is None or lse is None:
        with _on(stream):
            out = torch.empty(rows, heads, value, dtype=q.dtype, device=q.device) if out is None else out
            lse = torch.empty(rows, heads, dtype=torch.float32, device=q.device) if lse is None else lse
    if _rows(out, "out", value, device) != t or out.shape[:2] != q.shape[:2]:
        raise ValueError("out is [rows, heads, value] of q's type")
    if lse.get_device() != device or lse.dtype != torch.float32 or not lse.is_contiguous() or lse.shape != q.shape[:2]:
        raise ValueError("lse is fp32 [rows, heads]")
    rc = uzip_latent_attend_expanded(t, q.data_ptr(), q.stride(0), q.stride(1), rows, heads, k.data_ptr(), k.stride(0), k.stride(1),
                                     key_rot.data_ptr(), key_rot.stride(0), v.data_ptr(), v.stride(0), v.stride(1), keys, nope, rot, value,
                                     q_start.data_ptr(), k_start.data_ptr(), n, max_new, (nope + rot) ** -0.5 if scale is None else scale,
                                     out.data_ptr(), out.stride(0), out.stride(1), lse.data_ptr(), _handle(stream, device))
    if rc != OK:
        _check(rc, "uzip_latent_attend_expanded")
    _wrote(*given)
    return out, lse
