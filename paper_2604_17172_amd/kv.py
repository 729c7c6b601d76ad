"""Paged 8-bit key/value cache: binding of include/uzip_kv.h.

``KVCache`` holds a pool of pages; ``kv_plan`` gives a step's new tokens their
places, ``kv_store`` writes them, ``kv_attend`` lets them attend to their
requests' pages.  Outputs and workspaces that are not given are allocated with
torch; every call enqueues on ``stream`` or the current one.
"""
from __future__ import annotations

import contextlib
import ctypes

import torch

from . import BF16, E4M3FN, E5M2, EINVAL, FP16, FP32, OK, _check, _dev_empty, _lib, _stream

_c = ctypes
_vp, _u32, _i64, _sz, _int, _f32 = _c.c_void_p, _c.c_uint32, _c.c_int64, _c.c_size_t, _c.c_int, _c.c_float

KV_MAX_REQUESTS, KV_MAX_ROWS = 4096, 1 << 22


class uzip_kv_cache(_c.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_exp", _vp), ("v_exp", _vp), ("n_pages", _u32), ("n_heads", _u32),
                ("head_dim", _u32), ("page_tokens", _u32), ("dtype", _int)]


_cache_p = _c.POINTER(uzip_kv_cache)
_lib.uzip_kv_max_runs.argtypes = [_u32, _u32, _u32]
_lib.uzip_kv_max_runs.restype = _u32
_lib.uzip_kv_plan.argtypes = [_vp, _vp, _u32, _vp, _u32, _u32, _u32, _vp, _u32, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.uzip_kv_plan.restype = _int
_lib.uzip_kv_store.argtypes = [_cache_p, _int, _vp, _i64, _i64, _vp, _i64, _i64, _u32, _vp, _vp, _vp, _u32, _vp]
_lib.uzip_kv_store.restype = _int
_lib.uzip_kv_attend_workspace.argtypes = [_int, _u32, _u32, _u32, _u32, _u32, _u32]
_lib.uzip_kv_attend_workspace.restype = _sz
_lib.uzip_kv_attend.argtypes = [_cache_p, _int, _vp, _i64, _i64, _u32, _u32, _vp, _u32, _vp, _vp, _u32, _u32, _f32,
                                _u32, _vp, _i64, _i64, _vp, _vp, _sz, _vp]
_lib.uzip_kv_attend.restype = _int

EXPORTED = ["uzip_kv_max_runs", "uzip_kv_plan", "uzip_kv_store", "uzip_kv_attend_workspace", "uzip_kv_attend"]

uzip_kv_max_runs = _lib.uzip_kv_max_runs
uzip_kv_plan = _lib.uzip_kv_plan
uzip_kv_store = _lib.uzip_kv_store
uzip_kv_attend_workspace = _lib.uzip_kv_attend_workspace
uzip_kv_attend = _lib.uzip_kv_attend

_TYPES = {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32}
_CODES = {"e4m3fn": E4M3FN, "e5m2": E5M2, torch.float8_e4m3fn: E4M3FN, torch.float8_e5m2: E5M2,
          E4M3FN: E4M3FN, E5M2: E5M2}


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


class KVCache:
    """Pages of keys and values in 8 bits.

    k [pages, heads, page tokens, dim] and v [pages, heads, dim, page tokens],
    uint8 codes of ``dtype`` ("e4m3fn" or "e5m2"); k_exp and v_exp [pages, heads],
    uint8: a value is code * 2^(exponent - 127).
    """

    def __init__(self, k: torch.Tensor, k_exp: torch.Tensor, v: torch.Tensor, v_exp: torch.Tensor, dtype="e4m3fn"):
        _need(k.dim() == 4 and v.dim() == 4, "k and v have four dimensions")
        pages, heads, page, dim = k.shape
        _need(tuple(v.shape) == (pages, heads, dim, page), "v is k with its last two dimensions exchanged")
        _need(tuple(k_exp.shape) == tuple(v_exp.shape) == (pages, heads), "k_exp and v_exp are [pages, heads]")
        for x in (k, k_exp, v, v_exp):
            _need(x.is_cuda and x.device == k.device and x.is_contiguous() and x.element_size() == 1,
                  "the cache's arrays are contiguous bytes on one GPU")
        _need(dtype in _CODES, "dtype is e4m3fn or e5m2")
        self.k, self.k_exp, self.v, self.v_exp = k, k_exp, v, v_exp
        self.pages, self.heads, self.page_tokens, self.dim = pages, heads, page, dim
        self.code, self.device, self.index = _CODES[dtype], k.device, k.get_device()
        self.desc = uzip_kv_cache(k.data_ptr(), v.data_ptr(), k_exp.data_ptr(), v_exp.data_ptr(), pages, heads, dim, page,
                                  self.code)
        self._as_parameter_ = _c.byref(self.desc)

    @classmethod
    def empty(cls, pages: int, heads: int, dim: int, page_tokens: int = 64, dtype="e4m3fn", device="cuda") -> "KVCache":
        """A pool of unwritten pages."""
        def new(*shape):
            return torch.empty(*shape, dtype=torch.uint8, device=device)
        return cls(new(pages, heads, page_tokens, dim), new(pages, heads), new(pages, heads, dim, page_tokens),
                   new(pages, heads), dtype)


class KVPlan:
    """A step's places, on the GPU (see uzip_kv_plan), for up to ``requests`` requests and ``rows`` new tokens: lens
    int32 [requests], q_start int32 [requests + 1], slots int64 [rows], runs int32 [max runs, 2], counts int32 [2]
    (pages taken, runs), status int32 [1] (of the last call).  After a call with fewer requests or rows, lens, q_start
    and slots are the parts that it wrote."""

    __slots__ = ("requests", "rows", "page_tokens", "lens", "q_start", "slots", "runs", "counts", "status", "_ptrs", "_all")

    def __init__(self, requests: int, rows: int, page_tokens: int, device="cuda"):
        fits = 0 <= rows <= KV_MAX_ROWS and 0 <= requests <= KV_MAX_REQUESTS and 0 <= page_tokens < 1 << 32
        runs = uzip_kv_max_runs(rows, requests, page_tokens) if fits else 0
        if runs == 0:
            _check(EINVAL, "uzip_kv_max_runs")

        def new(*shape, dtype=torch.int32):
            return torch.empty(*shape, dtype=dtype, device=device)
        self.requests, self.rows, self.page_tokens = requests, rows, page_tokens
        self.lens, self.q_start, self.slots = new(requests), new(requests + 1), new(rows, dtype=torch.int64)
        self.runs, self.counts = new(runs, 2), new(2)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self._all = self.lens, self.q_start, self.slots
        self._ptrs = tuple(t.data_ptr() for t in (self.lens, self.q_start, self.slots, self.runs, self.counts, self.status))

    def _narrow(self, requests: int, rows: int) -> None:
        """What lies past a call's requests and rows is an earlier call's."""
        lens, q_start, slots = self._all
        self.lens, self.q_start, self.slots = lens[:requests], q_start[:requests + 1], slots[:rows]


def kv_plan_buffers(requests: int, rows: int, page_tokens: int, device="cuda") -> KVPlan:
    return KVPlan(requests, rows, page_tokens, device)


def _ints(x: torch.Tensor, name: str, device: int, dtype=torch.int32) -> None:
    if x.get_device() != device or x.dtype != dtype or not x.is_contiguous():
        raise ValueError(f"{name} is a contiguous {dtype} tensor on the current GPU")


# The current device and its stream's handle without making objects of them, which
# takes 3 us of a call that takes 4.
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _handle(stream, device: int) -> int:
    return _stream(stream) if stream is not None or _raw_stream is None else _raw_stream(device)


def _on(stream):
    """Where a call's own tensors are made: memory used on a stream has to be that stream's."""
    return torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext()


def kv_plan(old: torch.Tensor, new: torch.Tensor, free: torch.Tensor, table: torch.Tensor, page_tokens: int, rows: int,
            out: KVPlan | None = None, stream=None, check: bool = False) -> KVPlan:
    """Places for ``new[i]`` more tokens of requests that hold ``old[i]``: pages
    from the front of ``free`` go into ``table`` [requests, max pages].  With
    ``check`` the call waits for the GPU and raises UzipError where a request
    took no part."""
    device = _device()
    _ints(old, "old", device)
    _ints(new, "new", device)
    _ints(free, "free", device)
    _ints(table, "table", device)
    n = old.numel()
    if new.numel() != n or table.dim() != 2 or table.shape[0] != n:
        raise ValueError("old, new and table are of one batch")
    if out is None:
        with _on(stream):
            out = KVPlan(n, rows, page_tokens, old.device)
    elif (n > out.requests or not 0 <= rows <= out.rows or not out.page_tokens <= page_tokens < 1 << 32
          or out.lens.get_device() != device):
        raise ValueError("out is for fewer requests or rows, larger pages or another GPU")
    rc = uzip_kv_plan(old.data_ptr(), new.data_ptr(), n, free.data_ptr(), free.numel(), page_tokens, rows, table.data_ptr(),
                      table.shape[1], *out._ptrs, _handle(stream, device))
    if rc != OK:
        _check(rc, "uzip_kv_plan")
    if n != out.lens.numel() or rows != out.slots.numel():
        out._narrow(n, rows)
    if check:
        (stream or torch.cuda.current_stream()).synchronize()
        _check(int(out.status.item()), "uzip_kv_plan")
    return out


def _rows(x: torch.Tensor, name: str, dim: int, device: int) -> int:
    t = _TYPES.get(x.dtype)
    if t is None or x.get_device() != device or x.dim() != 3 or x.shape[2] != dim or (x.stride(2) != 1 and x.numel()):
        raise ValueError(f"{name} is [rows, heads, {dim}] in bf16, fp16 or fp32 with each head's values side by side")
    return t


def _current(cache: KVCache) -> int:
    device = _device()
    if cache.index != device:
        raise ValueError("the cache is on another GPU than the current one")
    return device


def kv_store(cache: KVCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, runs: torch.Tensor,
             counts: torch.Tensor, stream=None) -> None:
    """Write rows of k and v [rows, heads, dim] to the places that kv_plan made."""
    device = _current(cache)
    t = _rows(k, "k", cache.dim, device)
    if _rows(v, "v", cache.dim, device) != t or k.shape != v.shape or k.shape[1] != cache.heads:
        raise ValueError("k and v are [rows, the cache's heads, dim] of one type")
    _ints(slots, "slots", device, torch.int64)
    _ints(runs, "runs", device)
    _ints(counts, "counts", device)
    rows = k.shape[0]
    if slots.numel() < rows or counts.numel() < 2 or runs.numel() != 2 * runs.shape[0]:
        raise ValueError("slots has an entry for each row, runs two for each run, counts two")
    rc = uzip_kv_store(cache, t, k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1), rows,
                       slots.data_ptr(), runs.data_ptr(), counts.data_ptr(), runs.shape[0], _handle(stream, device))
    if rc != OK:
        _check(rc, "uzip_kv_store")


def kv_attend_workspace(q: torch.Tensor, cache: KVCache, requests: int, max_new: int) -> torch.Tensor:
    t = _rows(q, "q", cache.dim, cache.index)
    n = uzip_kv_attend_workspace(t, q.shape[0], q.shape[1], cache.heads, cache.dim, requests, max_new)
    if n == 0:
        _check(EINVAL, "uzip_kv_attend_workspace")
    return _dev_empty(n, q.device)


def kv_attend(q: torch.Tensor, cache: KVCache, table: torch.Tensor, lens: torch.Tensor, q_start: torch.Tensor,
              max_new: int, scale: float | None = None, window: int = 0, out: torch.Tensor | None = None,
              lse: torch.Tensor | None = None, ws: torch.Tensor | None = None, stream=None):
    """Causal attention of the new tokens q [rows, query heads, dim] over their
    requests' pages.  Returns (out like q, lse [rows, query heads] fp32)."""
    device = _current(cache)
    t = _rows(q, "q", cache.dim, device)
    rows, heads = q.shape[0], q.shape[1]
    n = lens.numel()
    _ints(table, "table", device)
    _ints(lens, "lens", device)
    _ints(q_start, "q_start", device)
    if table.dim() != 2 or table.shape[0] < n or q_start.numel() <= n:
        raise ValueError("table, lens and q_start are of one batch")
    if not (0 <= window < 1 << 32 and 0 <= max_new < 1 << 32):
        raise ValueError("window and max_new are not negative")
    if out is None or lse is None or ws is None:
        with _on(stream):
            out = torch.empty(rows, heads, cache.dim, dtype=q.dtype, device=q.device) if out is None else out
            lse = torch.empty(rows, heads, dtype=torch.float32, device=q.device) if lse is None else lse
            ws = kv_attend_workspace(q, cache, n, max_new) if ws is None else ws
    if _rows(out, "out", cache.dim, device) != t or out.shape != q.shape:
        raise ValueError("out is like q")
    if lse.get_device() != device or lse.dtype != torch.float32 or not lse.is_contiguous() or lse.shape != q.shape[:2]:
        raise ValueError("lse is fp32 [rows, query heads]")
    if ws.get_device() != device or not ws.is_contiguous():
        raise ValueError("ws is a contiguous tensor on the current GPU")
    rc = uzip_kv_attend(cache, t, q.data_ptr(), q.stride(0), q.stride(1), rows, heads, table.data_ptr(), table.shape[1],
                        lens.data_ptr(), q_start.data_ptr(), n, max_new, cache.dim ** -0.5 if scale is None else scale, window,
                        out.data_ptr(), out.stride(0), out.stride(1), lse.data_ptr(), ws.data_ptr(),
                        ws.numel() * ws.element_size(), _handle(stream, device))
    if rc != OK:
        _check(rc, "uzip_kv_attend")
    return out, lse
