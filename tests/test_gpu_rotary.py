"""GPU: rotary positions, their gradient, and turned keys into 8-bit pages, against oracle/rotary.py and
oracle/kv.py in 64 bits.

A turned value is off by oracle.rotary.error before it is rounded to its type (half an ulp); a code, whose only rounding
is its own, has to be the code of a value that far from the exact one, and a page's exponent likewise.
"""
import numpy as np
import pytest
import torch

from oracle import kv as ref_kv
from oracle import rotary as ref

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
U_OUT = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}
LEAST = {"bf16": 2.0 ** -130, "fp16": 2.0 ** -25, "fp32": 2.0 ** -130}


def say(*a):
    print("[rotary]", *a, flush=True)


@pytest.fixture(scope="module")
def uz():
    import paper_2604_17172_amd as m
    return m


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def ints(x):
    return dev(np.asarray(x, dtype=np.int32).reshape(np.shape(x)))


def np_of(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rows_of(shape, kind, g, how="", scale=1.0):
    """Values of a type: by themselves, a slice of a wider array ("fused"), or at odd strides ("odd")."""
    rows, heads, dim = shape
    x = torch.from_numpy(g.standard_normal(shape).astype(np.float32) * scale).to(TYPES[kind]).cuda()
    if how == "odd":
        wide = torch.full((rows, heads, dim + 3), 7.0, dtype=TYPES[kind], device="cuda")
        wide[:, :, 1:dim + 1] = x
        return wide[:, :, 1:dim + 1]
    if how == "fused":
        wide = torch.full((rows, heads + 2, dim), 7.0, dtype=TYPES[kind], device="cuda")
        wide[:, 1:heads + 1] = x
        return wide[:, 1:heads + 1]
    return x


def freq_of(rot, base=10000.0):
    return (base ** (-2.0 * np.arange(rot // 2) / rot)).astype(np.float32)


def check(got, x, places, freq, kind, **how):
    want = ref.rotate(np_of(x), places, freq, **how)
    tol = ref.error(np_of(x), places, freq, how.get("interleaved", False), how.get("first", 0), how.get("magnitude", 1.0))
    tol += U_OUT[kind] * (np.abs(want) + tol) + LEAST[kind]
    off = np.abs(np_of(got) - want)
    assert (off <= tol).all(), (np.argwhere(off > tol)[:4].tolist(), (off / tol).max())
    first, rot = how.get("first", 0), 2 * len(freq)                       # what is not turned keeps its bits
    for part in (slice(0, first), slice(first + rot, None)):
        assert torch.equal(got[..., part], x[..., part])


CASES = [  # rows, heads, dim, rot, first, interleaved, how
    (1, 1, 2, 2, 0, False, ""),
    (1, 1, 64, 64, 0, False, ""),
    (3, 2, 128, 128, 0, True, ""),
    (65, 14, 64, 32, 0, False, "fused"),
    (64, 32, 128, 128, 0, False, "fused"),
    (129, 3, 96, 48, 48, True, ""),
    (33, 5, 80, 20, 8, False, ""),
    (17, 2, 101, 38, 63, True, "odd"),
    (40, 7, 73, 14, 0, False, ""),
    (257, 1, 256, 256, 0, True, "odd"),
    (5, 300, 32, 16, 16, False, ""),
    (2, 2, 1024, 1024, 0, False, ""),
    (2000, 1, 64, 64, 0, True, ""),
    (1025, 4, 576, 64, 512, False, ""),
    (7, 2, 24, 16, 8, True, "fused"),
    (9, 3, 40, 32, 8, False, ""),
    (50, 3, 44, 24, 4, False, ""),
    (61, 3, 44, 24, 4, True, "fused"),
    (700, 5, 104, 40, 64, True, ""),
    (3, 2, 30, 12, 2, False, ""),
]


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_rotate(uz, case, kind):
    rows, heads, dim, rot, first, interleaved, how = case
    say("rotate", kind, case)
    g = np.random.default_rng(1)
    x = rows_of((rows, heads, dim), kind, g, how)
    places = g.integers(-5, 200000, rows).astype(np.int32)
    freq = freq_of(rot)
    for inverse, magnitude in [(False, 1.0), (True, 1.3)]:
        before = x.clone()
        out = rows_of((rows, heads, dim), kind, g, how)
        got = uz.rotate(x, ints(places), dev(freq), interleaved=interleaved, first=first, magnitude=magnitude, inverse=inverse, out=out)
        torch.cuda.synchronize()
        assert got is out and torch.equal(x, before)
        check(got, x, places, freq, kind, interleaved=interleaved, first=first, magnitude=magnitude, inverse=inverse)
        own = uz.rotate(x, ints(places), dev(freq), interleaved, first, magnitude, inverse)
        assert torch.equal(own, got)
        again = x.clone() if how == "" else x
        uz.rotate(again, ints(places), dev(freq), interleaved, first, magnitude, inverse, out=again)      # in place
        assert torch.equal(again, got)
        x.copy_(before)
    if how == "odd":                                                      # nothing beside the rows is written
        base = torch.as_strided(out, (rows, heads, dim + 3), out.stride(), out.storage_offset() - 1)
        assert (base[:, :, 0] == 7).all() and (base[:, :, dim + 1:] == 7).all()


def test_rotate_far_positions(uz):
    """Angles of millions of radians: 32 bits would lose them."""
    g = np.random.default_rng(2)
    places = np.array([2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 123456789, -7, 0], np.int32)
    x = rows_of((6, 2, 64), "fp32", g)
    freq = np.concatenate([freq_of(62), [np.float32(3.0)]]).astype(np.float32)
    got = uz.rotate(x, ints(places), dev(freq))
    check(got, x, places, freq, "fp32")
    assert torch.equal(got[5], x[5])


def test_rotate_of_nothing(uz):
    f, p = dev(freq_of(8)), ints([])
    assert uz.rotate(torch.zeros(0, 3, 8, device="cuda"), p, f).shape == (0, 3, 8)
    assert uz.rotate(torch.zeros(2, 0, 8, device="cuda"), ints([1, 2]), f).shape == (2, 0, 8)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
def test_rotate_gradients(uz, kind, interleaved):
    g = np.random.default_rng(3)
    rows, heads, dim, rot, first = 13, 3, 56, 24, 16
    places, freq = g.integers(0, 5000, rows).astype(np.int32), freq_of(24)
    x = rows_of((rows, heads, dim), kind, g).requires_grad_(True)
    y = uz.rotate(x, ints(places), dev(freq), interleaved, first, 1.25)
    assert y.requires_grad
    up = rows_of((rows, heads, dim), kind, g)
    grad, = torch.autograd.grad(y, x, up, create_graph=False)
    check(grad, up, places, freq, kind, interleaved=interleaved, first=first, magnitude=1.25, inverse=True)
    # a gradient that comes broadcast, and transposed
    s, = torch.autograd.grad(uz.rotate(x, ints(places), dev(freq), interleaved, first, 1.25).sum(), x)
    check(s, torch.ones_like(x), places, freq, kind, interleaved=interleaved, first=first, magnitude=1.25, inverse=True)
    t = rows_of((rows, dim, heads), kind, g).transpose(1, 2)
    d, = torch.autograd.grad(uz.rotate(x, ints(places), dev(freq), interleaved, first, 1.25), x, t)
    check(d, t, places, freq, kind, interleaved=interleaved, first=first, magnitude=1.25, inverse=True)
    if kind == "fp32":
        # differences: the operator is linear, so a step of 1 leaves only roundings, 2^-21 of the values here
        v = rows_of((rows, heads, dim), kind, g)
        with torch.no_grad():
            step = uz.rotate(x + v, ints(places), dev(freq), interleaved, first, 1.25) - y
        assert abs(float((step.double() * up.double()).sum() - (grad.double() * v.double()).sum())) < 2.0 ** -21 * 10 * step.numel() ** 0.5
        # the gradient of the gradient
        w = up.clone().requires_grad_(True)
        first_grad, = torch.autograd.grad(uz.rotate(x, ints(places), dev(freq), interleaved, first, 1.25), x, w, create_graph=True)
        second, = torch.autograd.grad(first_grad, w, v)
        check(second, v, places, freq, kind, interleaved=interleaved, first=first, magnitude=1.25)


def test_rotate_on_another_stream_and_in_a_graph(uz):
    g = np.random.default_rng(4)
    x, places, freq = rows_of((50, 4, 128), "bf16", g), ints(g.integers(0, 999, 50)), dev(freq_of(128))
    want = uz.rotate(x, places, freq)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = uz.rotate(x, places, freq, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    out = torch.zeros_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        uz.rotate(x, places, freq, out=out)
    for turn in range(3):
        x.copy_(rows_of((50, 4, 128), "bf16", g))
        places.copy_(ints(g.integers(0, 99999, 50)))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, uz.rotate(x, places, freq)), turn


def test_backward_in_a_graph_beside_an_eager_one(uz):
    """A captured forward and backward while an eager graph of the same leaf lives."""
    g = np.random.default_rng(5)
    leaf = rows_of((20, 2, 64), "fp32", g).requires_grad_(True)
    places, freq = ints(g.integers(0, 99, 20)), dev(freq_of(64))
    up = rows_of((20, 2, 64), "fp32", g)
    alive = uz.rotate(leaf, places, freq)
    grad = torch.zeros_like(up)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x = leaf.detach().requires_grad_(True)
        grad.copy_(torch.autograd.grad(uz.rotate(x, places, freq), x, up)[0])
    want, = torch.autograd.grad(alive, leaf, up)
    for _ in range(3):
        grad.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(grad, want)


# ------------------------------------------------------------------ places
@pytest.mark.parametrize("lens,new,pad", [([5], [1], 0), ([5, 0, 9], [2, 0, 9], 3), ([3, 7], [5, 1], 2), ([], [], 4), ([1] * 700, [1] * 700, 1)])
def test_positions(uz, lens, new, pad):
    q_start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    rows = int(q_start[-1]) + pad
    out = ints(np.full(rows + 2, 77))
    got = uz.kv_positions(ints(lens), ints(q_start), rows, out=out)
    assert np.array_equal(got[:rows].cpu().numpy(), ref.positions(lens, q_start, rows)) and (got[rows:] == 77).all()
    assert torch.equal(uz.kv_positions(ints(lens), ints(q_start), rows), got[:rows])


def test_positions_follow_the_plan(uz):
    """A refused request's rows have no place, and neither have rows past the last request."""
    old, new = [4, 10, 3], [2, 1, 3]
    table = ints(np.full((3, 1), -1))
    plan = uz.kv_plan(ints(old), ints(new), ints([0, 1, 2]), table, 16, 8)
    places = uz.kv_positions(plan.lens, plan.q_start, 8)
    assert places.tolist() == [4, 5, 10, 3, 4, 5, -1, -1]
    plan = uz.kv_plan(ints(old), ints([2, 60, 3]), ints([0, 1, 2]), table, 16, 70)
    assert uz.kv_positions(plan.lens, plan.q_start, 70).tolist() == [4, 5] + [-1] * 60 + [3, 4, 5] + [-1] * 5


# ------------------------------------------------------------------ turned keys into pages
STORES = [  # page, dim, heads, query heads, kind, fmt, old, new, rot, first, interleaved, how
    (16, 64, 1, 1, "bf16", "e4m3fn", [0], [1], 64, 0, False, ""),
    (64, 128, 2, 8, "bf16", "e4m3fn", [0, 3, 64, 63], [64, 5, 1, 2], 128, 0, False, "fused"),
    (16, 96, 3, 3, "fp16", "e5m2", [5, 0, 17], [40, 17, 15], 96, 0, True, ""),
    (256, 256, 1, 2, "fp32", "e4m3fn", [1, 255], [300, 2], 256, 0, False, ""),
    (32, 192, 2, 0, "fp32", "e5m2", [7, 31, 32], [1, 1, 1], 64, 128, False, ""),
    (128, 64, 2, 14, "fp16", "e4m3fn", [100, 1], [60, 128], 22, 5, True, "odd"),
    (256, 64, 5, 5, "bf16", "e5m2", [13], [511], 30, 0, False, "odd"),
    (16, 128, 4, 4, "fp32", "e4m3fn", [15, 16, 1], [3, 33, 0], 48, 16, True, "fused"),
    (64, 96, 6, 6, "bf16", "e4m3fn", [9, 70, 5, 1], [1, 1, 1, 1], 96, 0, True, ""),
    (64, 256, 3, 3, "bf16", "e4m3fn", [9, 70, 5, 1], [1, 1, 1, 1], 34, 101, False, ""),
]


@pytest.mark.parametrize("case", STORES, ids=str)
def test_rotate_store(uz, case):
    page, dim, heads, q_heads, kind, fmt, old, new, rot, first, interleaved, how = case
    say("store", case)
    g = np.random.default_rng(11)
    pages, freq = 40, freq_of(rot)
    u8 = lambda *s: g.integers(0, 255, s).astype(np.uint8)  # noqa: E731
    plain = lambda *s: u8(*s) & 0xBB  # noqa: E731  no NaN and no infinity in either format
    host = {"k": plain(pages, heads, page, dim), "v": plain(pages, heads, page, dim),
            "k_exp": (u8(pages, heads) % 40 + 100).astype(np.uint8), "v_exp": (u8(pages, heads) % 40 + 100).astype(np.uint8)}
    cache = uz.KVCache(dev(host["k"]), dev(host["k_exp"]), dev(host["v"].transpose(0, 1, 3, 2)), dev(host["v_exp"]), fmt)
    free = g.permutation(pages).astype(np.int32)
    table = np.full((len(old), 40), -1, np.int32)
    for i, o in enumerate(old):                                           # pages of what was there before
        n = -(-o // page)
        table[i, :n], free = free[:n], free[n:]
    rows = int(np.sum(new)) + 2                                           # and two rows of no request
    plan = uz.kv_plan(ints(old), ints(new), ints(free), ints(table), page, rows)
    want = ref_kv.plan(old, new, free, table, page, rows)
    places = uz.kv_positions(plan.lens, plan.q_start, rows)
    k, v = rows_of((rows, heads, dim), kind, g, how, 2.0), rows_of((rows, heads, dim), kind, g, how, 5.0)
    q = rows_of((rows, q_heads, dim), kind, g, how) if q_heads else None
    got = uz.kv_rotate_store(cache, k, v, places, dev(freq), plan.slots, plan.runs, plan.counts, q=q, interleaved=interleaved, first=first,
                             magnitude=1.1)
    torch.cuda.synchronize()
    at = ref.positions(want["lens"], want["q_start"], rows)
    if q is None:
        assert got is None
    else:
        check(got, q, at, freq, kind, interleaved=interleaved, first=first, magnitude=1.1)
    turned = ref.rotate(np_of(k), at, freq, interleaved, first, 1.1)
    off = ref.error(np_of(k), at, freq, interleaved, first, 1.1)
    ends = []
    for sign in (-1, 1):                                                  # the codes of the least and the largest it may be
        c, e = host["k"].copy(), host["k_exp"].copy()
        ref_kv.store(c, e, turned + sign * off, want["slots"], want["runs"], page, fmt)
        ends.append((c, e))
    have, have_e = cache.k.cpu().numpy(), cache.k_exp.cpu().numpy()
    assert ((have_e == ends[0][1]) | (have_e == ends[1][1])).all()
    same = (have_e == ends[0][1]) & (have_e == ends[1][1])
    assert same.mean() > 0.9
    ok = (have == ends[0][0]) | (have == ends[1][0])
    assert ok[same].all() and (ends[0][0] != ends[1][0]).mean() < 1e-3
    ref_kv.store(host["v"], host["v_exp"], np_of(v), want["slots"], want["runs"], page, fmt)
    assert np.array_equal(cache.v_exp.cpu().numpy(), host["v_exp"])
    assert np.array_equal(cache.v.cpu().numpy().transpose(0, 1, 3, 2), host["v"])


@pytest.mark.parametrize("fmt", ["e4m3fn", "e5m2"])
@pytest.mark.parametrize("how", ["", "odd"])
def test_rotate_store_of_special_values(uz, fmt, how):
    """NaN and infinities in the part that is not turned, and places that are none."""
    g = np.random.default_rng(12)
    page, dim, rows = 16, 64, 20
    cache = uz.KVCache.empty(3, 1, dim, page, fmt)
    for t in (cache.k, cache.v, cache.k_exp, cache.v_exp):
        t.fill_(9)
    k, v = rows_of((rows, 1, dim), "fp16", g, how), rows_of((rows, 1, dim), "fp16", g, how)
    k[2, 0, 40], k[3, 0, 41], k[3, 0, 42] = float("nan"), float("inf"), float("-inf")
    slots = torch.arange(rows, device="cuda") + 16                        # pages 1 and 2
    slots[16:] = -1
    runs, counts = ints([[0, 16], [16, 4], [50, 1], [-3, 2]]), ints([0, 4])
    places = ints(np.zeros(rows))
    uz.kv_rotate_store(cache, k, v, places, dev(freq_of(32)), slots, runs, counts)
    codes = cache.k.cpu().numpy()
    assert (codes[0] == 9).all() and (codes[2] == 9).all() and (cache.v[2] == 9).all()
    want = np.full((3, 1, page, dim), 9, np.uint8)
    e = np.full((3, 1), 9, np.uint8)
    ref_kv.store(want, e, np_of(k), slots.cpu().numpy(), [(0, 16)], page, fmt)
    assert np.array_equal(codes, want) and np.array_equal(cache.k_exp.cpu().numpy(), e)


def test_refusals(uz):
    x, f, p = torch.zeros(4, 2, 64, device="cuda"), dev(freq_of(64)), ints([0, 1, 2, 3])
    bad = [dict(x=x[0]), dict(x=x.double()), dict(x=x[..., ::2]), dict(x=x.cpu()), dict(p=p[:3]), dict(p=p.long()), dict(p=p.cpu()),
           dict(f=f.double()), dict(f=f[::2]), dict(f=dev(freq_of(66))), dict(f=f[:0]), dict(f=f[None]), dict(first=2), dict(first=-1),
           dict(out=x.half()), dict(out=x[:2]), dict(f=f.cpu())]
    for b in bad:
        a = {"x": x, "p": p, "f": f, "first": 0, "out": None, **b}
        with pytest.raises(ValueError):
            uz.rotate(a["x"], a["p"], a["f"], first=a["first"], out=a["out"])
    with pytest.raises(uz.UzipError):
        uz.rotate(x, p, f, magnitude=float("nan"))
    leaf = x.clone().requires_grad_(True)
    with pytest.raises(ValueError):
        uz.rotate(leaf, p, f, out=torch.empty_like(x))
    with pytest.raises(ValueError):
        uz.rotate(leaf, p, f, stream=torch.cuda.Stream())
    with pytest.raises(ValueError):
        uz.kv_positions(p, p, 4)
    with pytest.raises(ValueError):
        uz.kv_positions(p[:3], p, 4, out=p[:2])
    cache = uz.KVCache.empty(2, 2, 64, 16)
    slots, runs, counts = torch.zeros(4, dtype=torch.int64, device="cuda"), ints([[0, 1]]), ints([0, 0])
    k = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    for b in [dict(k=k[:, :1]), dict(q=k[:2]), dict(q=k.float()), dict(q_out=k), dict(q=k, q_out=k[:, :1]), dict(f=dev(freq_of(66))), dict(first=1),
              dict(slots=slots[:2]), dict(q=k.clone().requires_grad_(True)), dict(k=k.clone().requires_grad_(True))]:
        a = {"k": k, "q": None, "q_out": None, "f": f, "first": 0, "slots": slots, **b}
        with pytest.raises(ValueError):
            uz.kv_rotate_store(cache, a["k"], k, p, a["f"], a["slots"], runs, counts, q=a["q"], q_out=a["q_out"], first=a["first"])
    with torch.no_grad():                                                 # what a server's call looks like
        uz.kv_rotate_store(cache, k, k, p, f, slots, runs, counts, q=k.clone().requires_grad_(True))
