"""Rotary positions and the latent cache without a GPU: the library exports what the headers declare, refuses what they
forbid before any GPU call, and the oracles agree with differences and with each other."""
import ctypes as c
import os
import re

import numpy as np
import pytest
import torch

from oracle import latent as ref_latent
from oracle import rotary as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def uz():
    import paper_2604_17172_amd as m
    return m


@pytest.mark.parametrize("header,module", [("uzip_rotary.h", "rotary"), ("uzip_latent.h", "latent")])
def test_exports(uz, header, module):
    import importlib
    mod = importlib.import_module(f"paper_2604_17172_amd.{module}")
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    names = set(re.findall(r"\b(uzip_[a-z_]+)\s*\(", text))
    assert names == set(mod.EXPORTED) and all(hasattr(uz._lib, n) for n in names)


def turn(uz, **k):
    a = dict(positions=4096, freq=4096, rot=64, first=0, interleaved=0, inverse=0, magnitude=1.0)
    return c.byref(uz.uzip_turn(*{**a, **k}.values()))


def test_rotate_refuses(uz):
    def call(dtype=0, x=4096, xr=128, xh=64, rows=4, heads=2, dim=64, t=None, out=8192, o_r=128, oh=64):
        return uz.uzip_rotate(dtype, x, xr, xh, rows, heads, dim, t or turn(uz), out, o_r, oh, None)
    bad = [dict(dtype=3), dict(dtype=9), dict(x=None), dict(x=4097), dict(out=None), dict(out=8193), dict(rows=(1 << 22) + 1), dict(heads=65536),
           dict(dim=63), dict(dim=1025), dict(xr=1 << 40), dict(oh=-(1 << 40)), dict(rows=1 << 22, heads=17), dict(dtype=2, x=4098)]
    bad += [dict(t=turn(uz, **k)) for k in (dict(rot=0), dict(rot=63), dict(rot=1026), dict(first=1), dict(first=2000), dict(interleaved=2), dict(inverse=2),
                                            dict(magnitude=float("inf")), dict(magnitude=float("nan")), dict(positions=None), dict(freq=None),
                                            dict(positions=4098), dict(freq=4097))]
    for b in bad:
        assert call(**b) == uz.EINVAL, b
    assert uz.uzip_rotate(0, 4096, 128, 64, 4, 2, 64, None, 8192, 128, 64, None) == uz.EINVAL
    assert call(rows=0) == uz.OK and call(heads=0) == uz.OK


def test_positions_refuses(uz):
    assert uz.uzip_kv_positions(64, 64, 4097, 4, 64, None) == uz.EINVAL
    assert uz.uzip_kv_positions(64, 64, 1, (1 << 22) + 1, 64, None) == uz.EINVAL
    for args in [(None, 64, 1, 4, 64), (64, None, 1, 4, 64), (64, 64, 1, 4, None), (65, 64, 1, 4, 64), (64, 66, 1, 4, 64), (64, 64, 1, 4, 65)]:
        assert uz.uzip_kv_positions(*args, None) == uz.EINVAL
    assert uz.uzip_kv_positions(None, None, 0, 0, None, None) == uz.OK


def test_rotate_store_refuses(uz):
    good = uz.uzip_kv_cache(4096, 4096, 4096, 4096, 8, 2, 64, 16, uz.E4M3FN)

    def call(cache=good, dtype=0, k=4096, v=4096, rows=4, slots=4096, runs=4096, counts=4096, max_runs=2, t=None, q=4096, heads=4, out=8192, qr=256):
        return uz.uzip_kv_rotate_store(c.byref(cache), dtype, k, 128, 64, v, 128, 64, rows, slots, runs, counts, max_runs, t or turn(uz), q, qr, 64,
                                       heads, out, 256, 64, None)
    other = lambda **k: uz.uzip_kv_cache(*{**dict(k=4096, v=4096, ke=4096, ve=4096, n=8, h=2, d=64, p=16, t=3), **k}.values())  # noqa: E731
    bad = [dict(cache=other(d=80)), dict(cache=other(p=24)), dict(cache=other(n=0)), dict(cache=other(t=0)), dict(cache=other(k=4100)), dict(dtype=4),
           dict(k=None), dict(v=4097), dict(rows=(1 << 22) + 1), dict(slots=None), dict(slots=4100), dict(runs=None), dict(counts=None), dict(counts=4098),
           dict(max_runs=(1 << 22) + 1), dict(q=None), dict(out=None), dict(q=4097), dict(qr=1 << 40)]
    bad += [dict(t=turn(uz, **k)) for k in (dict(inverse=1), dict(rot=66), dict(first=2), dict(positions=None), dict(freq=None), dict(rot=3))]
    for b in bad:
        assert call(**b) == uz.EINVAL, b
    assert call(rows=0) == uz.OK and call(max_runs=0, heads=0) == uz.OK


def latent_cache(uz, **k):
    return c.byref(uz.uzip_latent_cache(*{**dict(codes=4096, exps=4096, n=8, latent=512, rot=64, page=16, t=uz.E4M3FN), **k}.values()))


BAD_CACHES = [dict(codes=None), dict(codes=4100), dict(exps=None), dict(exps=4097), dict(n=0), dict(latent=384), dict(latent=0), dict(rot=48), dict(rot=0),
              dict(page=8), dict(page=512), dict(page=24), dict(t=0), dict(n=1 << 27)]


def test_latent_store_refuses(uz):
    def call(cache=None, dtype=0, x=4096, xr=512, r=4096, rr=64, rows=4, slots=4096, t=None, q=4096, heads=2, out=8192):
        return uz.uzip_latent_store(cache or latent_cache(uz), dtype, x, xr, r, rr, rows, slots, t or turn(uz), q, 128, 64, heads, out, 128, 64, None)
    bad = [dict(cache=latent_cache(uz, **k)) for k in BAD_CACHES]
    bad += [dict(dtype=3), dict(x=None), dict(x=4097), dict(r=None), dict(xr=1 << 40), dict(rr=-(1 << 40)), dict(rows=(1 << 22) + 1), dict(slots=None),
            dict(slots=4100), dict(q=None), dict(out=None)]
    bad += [dict(t=turn(uz, **k)) for k in (dict(inverse=1), dict(rot=32), dict(first=8), dict(positions=None), dict(freq=4098))]
    for b in bad:
        assert call(**b) == uz.EINVAL, b
    assert call(rows=0) == uz.OK
    assert uz.uzip_latent_store(None, 0, 4096, 512, 4096, 64, 4, 4096, turn(uz), None, 0, 0, 0, None, 0, 0, None) == uz.EINVAL


def test_latent_attend_refuses(uz):
    size = uz.uzip_latent_attend_workspace
    assert size(512, 4, 2, 1, 1) > 0 and size(256, 0, 1, 0, 0) > 0
    for args in [(384, 4, 2, 1, 1), (512, (1 << 22) + 1, 1, 1, 1), (512, 4, 0, 1, 1), (512, 4, 1025, 1, 1), (512, 4, 2, 4097, 1), (512, 1 << 22, 17, 1, 1)]:
        assert size(*args) == 0
    most = size(512, 64, 128, 64, 1)

    def call(cache=None, dtype=0, q=4096, qr=1152, rows=64, heads=128, table=4096, pages=4, lens=4096, start=4096, reqs=64, scale=0.1, out=4096, lse=None,
             ws=4096, ws_bytes=most):
        return uz.uzip_latent_attend(cache or latent_cache(uz), dtype, q, qr, 576, rows, heads, table, pages, lens, start, reqs, 1, scale, out, 1024, 512, lse,
                                     ws, ws_bytes, None)
    bad = [dict(cache=latent_cache(uz, **k)) for k in BAD_CACHES]
    bad += [dict(dtype=2), dict(dtype=3), dict(q=None), dict(q=4097), dict(qr=1 << 40), dict(heads=0), dict(heads=1025), dict(table=None), dict(table=4098),
            dict(lens=None), dict(start=None), dict(start=4097), dict(reqs=4097), dict(scale=float("nan")), dict(scale=float("inf")), dict(out=None),
            dict(lse=4098), dict(ws=4104), dict(pages=1 << 31), dict(rows=(1 << 22) + 1)]
    for b in bad:
        assert call(**b) == uz.EINVAL, b
    assert call(ws=None) == uz.ENOSPC and call(ws_bytes=most - 1) == uz.ENOSPC and call(rows=0) == uz.OK


def test_expanded_refuses(uz):
    def call(dtype=0, q=4096, rows=4, heads=2, k=4096, kr=128, r=4096, v=4096, keys=4, nope=64, rot=32, value=64, qs=4096, ks=4096, reqs=1, scale=0.1,
             out=4096, lse=None):
        return uz.uzip_latent_attend_expanded(dtype, q, 192, 96, rows, heads, k, kr, 64, r, 32, v, 128, 64, keys, nope, rot, value, qs, ks, reqs, 4, scale,
                                              out, 128, 64, lse, None)
    for b in [dict(dtype=2), dict(q=None), dict(q=4097), dict(heads=0), dict(heads=1025), dict(k=None), dict(kr=1 << 40), dict(r=None), dict(v=4097),
              dict(nope=96), dict(nope=0), dict(rot=16), dict(value=96), dict(qs=None), dict(ks=None), dict(ks=4098), dict(reqs=4097), dict(out=None),
              dict(lse=4098), dict(scale=float("nan")), dict(rows=(1 << 22) + 1), dict(keys=(1 << 22) + 1), dict(rows=1 << 22, heads=17)]:
        assert call(**b) == uz.EINVAL, b
    assert call(rows=0) == uz.OK


# ------------------------------------------------------------------ frequencies
def test_frequencies(uz):
    f, m = uz.rotary_frequencies(8, 10000.0, device="cpu")
    assert torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001])) and m == 1.0 and f.dtype == torch.float32
    g, m = uz.rotary_frequencies(8, 10000.0, "linear", 4.0, device="cpu")
    assert torch.allclose(g, f / 4) and m == 1.0
    g, m = uz.rotary_frequencies(8, 10000.0, "base", 4.0, device="cpu")
    assert g[0] == 1 and abs(float(g[-1] / f[-1]) - 0.25) < 1e-6 and m == 1.0
    f, _ = uz.rotary_frequencies(128, 10000.0, device="cpu")
    g, m = uz.rotary_frequencies(128, 10000.0, "parts", 8.0, 4096, device="cpu")
    turns = 4096 * f / (2 * np.pi)
    ratio = g / f
    assert (ratio[turns > 40] == 1).all() and torch.allclose(ratio[turns < 0.8], torch.tensor(0.125)) and (ratio[1:] <= ratio[:-1]).all()
    assert abs(m - (0.1 * np.log(8) + 1)) < 1e-12
    for args in [(7,), (0,), (8, 1.0), (8, 1e4, "linear", 0.5), (8, 1e4, "more"), (8, 1e4, "parts", 2.0), (8, 1e4, "parts", 2.0, 100, 1.0, 2.0)]:
        with pytest.raises(ValueError):
            uz.rotary_frequencies(*args, device="cpu")


@pytest.mark.parametrize("rot,trained", [(64, 131072), (128, 131072), (64, 65536), (96, 1 << 20), (64, 4096), (32, 1 << 22)])
def test_frequencies_of_long_trained_contexts(uz, rot, trained):
    """The slowest pairs turn more than once over the trained length: none of them is divided by the whole factor."""
    factor, base = 4.0, 10000.0
    plain, _ = uz.rotary_frequencies(rot, base, device="cpu")
    got, _ = uz.rotary_frequencies(rot, base, "parts", factor, trained, device="cpu")
    turns = [trained * base ** (-2 * i / rot) / (2 * np.pi) for i in range(rot // 2)]

    def number(t):                                                        # trained * base^(-2 n / rot) = 2 pi t
        return rot / 2 * np.log(trained / (2 * np.pi * t)) / np.log(base)
    low, high = max(np.floor(number(32)), 0), np.ceil(number(1))
    for i in range(rot // 2):
        part = min(max((i - low) / (high - low), 0), 1)
        ratio = float(got[i] / plain[i])
        assert abs(ratio - (1 - part + part / factor)) < 2.0 ** -22
        assert ratio > 1 / factor + 1e-3 or turns[i] < 1


# ------------------------------------------------------------------ the oracles
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_its_inverse_is_its_gradient(interleaved):
    g = np.random.default_rng(0)
    x, up = g.standard_normal((5, 2, 24)), g.standard_normal((5, 2, 24))
    places, freq = g.integers(0, 999, 5), np.array([1.0, 0.3, 0.01])
    y = ref.rotate(x, places, freq, interleaved, 4, 1.0)
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-13)
    assert np.allclose(ref.rotate(y, places, freq, interleaved, 4, 1.0, True), x, atol=1e-13)
    grad = ref.rotate(up, places, freq, interleaved, 4, 1.5, True)
    for _ in range(6):                                                    # differences
        d = g.standard_normal(x.shape) * 1e-4
        a, b = (float((ref.rotate(x + s * d, places, freq, interleaved, 4, 1.5) * up).sum()) for s in (1, -1))
        assert abs((a - b) / 2 - float((grad * d).sum())) < 1e-11


def test_both_forms_of_latent_attention_agree():
    g = np.random.default_rng(1)
    heads, nope, rot, value, latent, page = 3, 8, 4, 6, 16, 4
    codes, exps = (g.integers(0, 256, (6, page, latent + rot)) & 0xBB).astype(np.uint8), g.integers(120, 125, (6, page, 2)).astype(np.uint8)
    table, lens, q_start = np.array([[3, 1, 0], [5, 2, -1]]), [10, 7], [0, 3, 5]
    up_k, up_v = g.standard_normal((heads, nope, latent)), g.standard_normal((heads, value, latent))
    q = g.standard_normal((5, heads, nope + rot))
    absorbed = np.concatenate([np.einsum("rhn,hnl->rhl", q[..., :nope], up_k), q[..., nope:]], axis=-1)
    a = ref_latent.attend(absorbed, codes, exps, latent, "e4m3fn", table, lens, q_start, page, 0.01)
    from oracle.kv import decode
    rows = [codes[table[i, t // page], t % page] for i in range(2) for t in range(lens[i])]
    es = np.array([exps[table[i, t // page], t % page] for i in range(2) for t in range(lens[i])]).astype(float)
    x = decode(np.array(rows), "e4m3fn") * np.repeat(2.0 ** (es - 127), [latent, rot], axis=1)
    k, v = np.einsum("tl,hnl->thn", x[:, :latent], up_k), np.einsum("tl,hvl->thv", x[:, :latent], up_v)
    e = ref_latent.expanded(q, k, x[:, latent:], v, q_start, [0, 10, 17], 0.01)
    assert np.allclose(a["lse"], e["lse"], rtol=1e-12) and np.allclose(np.einsum("rhl,hvl->rhv", a["out"], up_v), e["out"], rtol=1e-9, atol=1e-12)


# ------------------------------------------------------------------ autograd
def test_calls_that_serve_refuse_what_autograd_follows(uz):
    import torch.autograd.forward_ad as fw
    from paper_2604_17172_amd.rotary import _serves
    x = torch.zeros(3)
    _serves(x, None)
    with pytest.raises(ValueError, match="no gradient"):
        _serves(None, x.clone().requires_grad_(True))
    with torch.no_grad():
        _serves(x.clone().requires_grad_(True))
    with fw.dual_level():
        _serves(x)
        for grad in (torch.enable_grad, torch.no_grad):
            with grad(), pytest.raises(ValueError, match="no gradient"):
                _serves(fw.make_dual(x, x))


def test_rotate_refuses_frequencies_that_are_learned(uz):
    import torch.autograd.forward_ad as fw
    x, places, freq = torch.zeros(2, 1, 8), torch.zeros(2, dtype=torch.int32), torch.ones(4)
    with pytest.raises(ValueError, match="frequencies"):
        uz.rotate(x, places, freq.clone().requires_grad_(True))
    with fw.dual_level(), pytest.raises(ValueError, match="frequencies"):
        uz.rotate(x, places, fw.make_dual(freq, freq))


def test_outputs_whose_rows_share_memory(uz):
    from paper_2604_17172_amd.kv import _apart
    x = torch.zeros(3, 2, 8)
    for good in (None, x, x[:, :1], x[:1].expand(1, 2, 8), torch.zeros(3, 1, 8).expand(3, 1, 8), x[:0], x.transpose(0, 1)):
        _apart(good, "out")
    for bad in (x[:1].expand(3, 2, 8), x[:, :1].expand(3, 2, 8)):
        with pytest.raises(ValueError, match="lie on one another"):
            _apart(bad, "out")
