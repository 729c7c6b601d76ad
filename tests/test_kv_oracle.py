"""The plain definitions of the paged 8-bit cache (oracle/kv.py) against facts
known otherwise, and the host-side checks of the library's entry points (no GPU
is touched: every call here returns before the library makes any HIP call)."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from oracle import kv as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TORCH = {"e4m3fn": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.fixture(scope="module")
def uz():
    import paper_2604_17172_amd as m
    return m


@pytest.mark.parametrize("fmt", ["e4m3fn", "e5m2"])
def test_code_values_are_torchs(fmt):
    want = torch.arange(256, dtype=torch.uint8).view(TORCH[fmt]).double().numpy()
    assert np.array_equal(ref.code_values(fmt), want, equal_nan=True)


@pytest.mark.parametrize("fmt", ["e4m3fn", "e5m2"])
def test_encode_rounds_to_nearest_even(fmt):
    g = np.random.default_rng(3)
    top = ref.FORMATS[fmt][2]
    values = ref.code_values(fmt)
    finite = np.sort(values[np.isfinite(values)])
    x = np.concatenate([g.standard_normal(20000) * 10, g.uniform(-top, top, 20000), values, (finite[1:] + finite[:-1]) / 2,
                        g.standard_normal(2000) * 2.0 ** -9]).astype(np.float32)
    x = x[np.abs(x) <= top]
    want = torch.from_numpy(x).to(TORCH[fmt]).view(torch.uint8).numpy()
    assert np.array_equal(ref.encode(x, fmt), want)
    assert np.array_equal(ref.encode([top * 1.5, -1e30], fmt), ref.encode([top, -top], fmt))
    special = ref.encode([np.inf, -np.inf, np.nan], fmt).tolist()
    assert special == ([0x7F, 0xFF, 0x7F] if fmt == "e4m3fn" else [0x7C, 0xFC, 0x7F])


@pytest.mark.parametrize("fmt,top", [("e4m3fn", 448.0), ("e5m2", 57344.0)])
def test_exponents(fmt, top):
    assert ref.exponent(top, fmt) == 127 and ref.exponent(np.nextafter(top, 1e9), fmt) == 128
    assert ref.exponent(top / 2, fmt) == 126 and ref.exponent(0.0, fmt) == 27
    big = float(np.finfo(np.float32).max)
    e = ref.exponent(big, fmt)
    assert e == ref.FORMATS[fmt][3] and top * 2.0 ** (e - 127) < big      # the largest scaled code is finite


def test_plan_by_hand():
    table = np.full((3, 4), -1, np.int32)
    table[0, 0] = 9
    p = ref.plan([3, 0, 16], [15, 1, 0], [5, 6, 7], table, 16, 17)
    assert p["table"].tolist() == [[9, 5, -1, -1], [6, -1, -1, -1], [-1, -1, -1, -1]]
    assert p["lens"].tolist() == [18, 1, 16] and p["q_start"].tolist() == [0, 15, 16, 16]
    assert p["slots"].tolist() == [9 * 16 + i for i in range(3, 16)] + [80, 81, 96, -1]
    assert p["runs"].tolist() == [[0, 13], [13, 2], [15, 1]] and p["counts"].tolist() == [2, 3] and p["status"] == 0


def test_attend_by_hand():
    """One head of two channels in effect: the weights follow from the scores by hand."""
    k = np.zeros((1, 1, 16, 64), np.uint8)
    v = np.zeros((1, 1, 16, 64), np.uint8)
    one = int(ref.encode(1.0, "e4m3fn"))
    k[0, 0, 0, 0] = k[0, 0, 1, 1] = v[0, 0, 0, 0] = v[0, 0, 1, 1] = one
    q = np.zeros((2, 1, 64))
    q[:, 0, 0] = np.log(3.0)
    e = np.full((1, 1), 128, np.uint8)                                    # scale 2
    r = ref.attend(q, k, e, v, e, "e4m3fn", np.array([[0]]), [2], [0, 2], 16, 0.5)
    assert np.allclose(r["out"][0, 0, :2], [2, 0]) and np.allclose(r["out"][1, 0, :2], [1.5, 0.5])
    assert np.allclose(r["lse"][:, 0], [np.log(3), np.log(4)])
    r = ref.attend(q, k, e, v, e, "e4m3fn", np.array([[0]]), [2], [0, 2], 16, 0.5, window=1)
    assert np.allclose(r["out"][1, 0, :2], [0, 2])


# ------------------------------------------------------------------ host side of the library
def test_library_exports_every_declared_symbol(uz):
    text = open(os.path.join(ROOT, "include", "uzip_kv.h")).read()
    names = set(re.findall(r"\b(uzip_kv_[a-z_]+)\s*\(", text))
    from paper_2604_17172_amd import kv
    assert names == set(kv.EXPORTED)
    for name in names:
        assert hasattr(uz._lib, name), name


def test_max_runs(uz):
    for rows, reqs, page in [(0, 0, 16), (1, 1, 64), (64, 64, 64), (65536, 1024, 16), (8192, 1, 256), (5, 4096, 32)]:
        assert uz.uzip_kv_max_runs(rows, reqs, page) == ref.max_runs(rows, reqs, page)
    assert uz.uzip_kv_max_runs(1, 1, 48) == 0 and uz.uzip_kv_max_runs(1, 1, 8) == 0 and uz.uzip_kv_max_runs(1, 1, 512) == 0
    assert uz.uzip_kv_max_runs(1, 4097, 16) == 0 and uz.uzip_kv_max_runs((1 << 22) + 1, 1, 16) == 0


def cache_desc(uz, **kw):
    a = {"k": 4096, "v": 8192, "k_exp": 1, "v_exp": 1, "n_pages": 4, "n_heads": 2, "head_dim": 128, "page_tokens": 64,
         "dtype": uz.E4M3FN, **kw}
    return uz.uzip_kv_cache(*[a[f] for f, _ in uz.uzip_kv_cache._fields_])


BAD_CACHES = [dict(k=None), dict(v=8200), dict(k=4104), dict(k_exp=None), dict(v_exp=None), dict(n_pages=0), dict(n_heads=0),
              dict(head_dim=80), dict(head_dim=0), dict(head_dim=512), dict(page_tokens=8), dict(page_tokens=48),
              dict(page_tokens=512), dict(dtype=0), dict(dtype=7), dict(n_pages=1 << 27, page_tokens=16)]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=lambda d: ",".join(f"{k}={v}" for k, v in d.items()))
def test_bad_caches_are_refused(uz, bad):
    c = ctypes.byref(cache_desc(uz, **bad))
    assert uz.uzip_kv_store(c, 0, 64, 256, 128, 64, 256, 128, 1, 64, 64, 64, 1, None) == uz.EINVAL
    assert uz.uzip_kv_attend(c, 0, 64, 256, 128, 1, 2, 64, 1, 64, 64, 1, 1, 1.0, 0, 64, 256, 128, 64, 64, 1 << 30,
                             None) == uz.EINVAL


def test_store_refusals(uz):
    c = ctypes.byref(cache_desc(uz))
    good = [c, 0, 64, 256, 128, 64, 256, 128, 1, 64, 64, 64, 1, None]

    def call(**at):
        a = list(good)
        for i, x in at.items():
            a[int(i[1:])] = x
        return uz.uzip_kv_store(*a)
    assert uz.uzip_kv_store(None, *good[1:]) == uz.EINVAL
    for at, x in [(1, 3), (1, -1), (2, None), (2, 65), (5, 65), (5, None), (3, 1 << 40), (7, -(1 << 40)), (8, (1 << 22) + 1),
                  (9, None), (9, 68), (10, None), (10, 66), (11, None), (11, 66)]:
        assert call(**{f"a{at}": x}) == uz.EINVAL, (at, x)
    assert call(a8=0) == uz.OK and call(a12=0) == uz.OK                   # nothing to store


def test_plan_refusals(uz):
    good = [64, 64, 2, 64, 8, 64, 10, 64, 4, 128, 64, 64, 64, 64, None, None]

    def call(**at):
        a = list(good)
        for i, x in at.items():
            a[int(i[1:])] = x
        return uz.uzip_kv_plan(*a)
    assert call(a9=64) == uz.EINVAL                                       # lengths out over lengths in
    for at, x in [(0, None), (0, 66), (1, None), (1, 66), (2, 4097), (3, None), (3, 66), (4, 1 << 31), (5, 24), (5, 0),
                  (6, (1 << 22) + 1), (7, None), (7, 66), (8, 1 << 31), (9, None), (9, 66), (10, None), (10, 66), (11, None),
                  (11, 68), (12, None), (12, 66), (13, None), (13, 66), (14, 66)]:
        assert call(**{f"a{at}": x}) == uz.EINVAL, (at, x)


def test_attend_refusals(uz):
    c = ctypes.byref(cache_desc(uz))
    ws = uz.uzip_kv_attend_workspace(0, 1, 4, 2, 128, 1, 1)
    assert ws > 0
    good = [c, 0, 64, 512, 128, 1, 4, 64, 1, 64, 64, 1, 1, 1.0, 0, 64, 512, 128, 64, 64, ws, None]

    def call(**at):
        a = list(good)
        for i, x in at.items():
            a[int(i[1:])] = x
        return uz.uzip_kv_attend(*a)
    assert uz.uzip_kv_attend(None, *good[1:]) == uz.EINVAL
    for at, x in [(1, 3), (1, -1), (2, None), (2, 65), (3, 1 << 40), (5, (1 << 22) + 1), (5, 1 << 25), (6, 0), (6, 3), (6, 1 << 27), (7, None),
                  (7, 66), (8, 1 << 31), (9, None), (9, 66), (10, None), (10, 66), (11, 4097), (13, float("nan")),
                  (13, float("inf")), (15, None), (15, 65), (18, 66), (19, 72)]:
        assert call(**{f"a{at}": x}) == uz.EINVAL, (at, x)
    assert call(a19=None) == uz.ENOSPC and call(a20=ws - 1) == uz.ENOSPC
    assert call(a5=0) == uz.OK                                            # no rows
    for bad in [(3, 1, 4, 2, 128, 1, 1), (0, 1, 4, 3, 128, 1, 1), (0, 1, 4, 0, 128, 1, 1), (0, 1, 0, 2, 128, 1, 1),
                (0, 1, 4, 2, 100, 1, 1), (0, (1 << 22) + 1, 4, 2, 128, 1, 1), (0, 1, 4, 2, 128, 4097, 1)]:
        assert uz.uzip_kv_attend_workspace(*bad) == 0, bad
