"""GPU: pages, store and attention of the 8-bit key/value cache against the
64-bit definitions in oracle/kv.py.

plan and store give whole numbers and bytes: they have to be equal.  Attention's
tolerance for each output follows from what is rounded: the output itself to its
type (half an ulp), each probability to U_P, each score by its products' sums
(dim * 2^-24 of the sum of magnitudes) and by the exponential (2^-22 of the score
and 2^-21), and the row's sum (tokens * 2^-24); probabilities err by twice
that, in the numerator and in the sum.
"""
import numpy as np
import pytest
import torch

from oracle import kv as ref

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
U_OUT = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}       # half an ulp at the low end of a binade
U_P = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -16, "fp32": 2.0 ** -24}         # the same of 8, 16 and 24 bits


def say(*a):
    print("[kv]", *a, flush=True)


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
    return t.float().cpu().numpy().astype(np.float64)


# ------------------------------------------------------------------ plan
def check_plan(uz, old, new, free, table, page, rows):
    say("plan", len(old), "requests", rows, "rows", "page", page)
    want = ref.plan(old, new, free, np.asarray(table, np.int32), page, rows)
    t = ints(table)
    got = uz.kv_plan(ints(old), ints(new), ints(free), t, page, rows)
    torch.cuda.synchronize()
    assert np.array_equal(t.cpu().numpy(), want["table"])
    assert np.array_equal(got.lens.cpu().numpy(), want["lens"])
    assert np.array_equal(got.q_start.cpu().numpy(), want["q_start"])
    assert np.array_equal(got.slots.cpu().numpy(), want["slots"])
    assert np.array_equal(got.counts.cpu().numpy(), want["counts"])
    n = len(want["runs"])
    assert np.array_equal(got.runs[:n].cpu().numpy(), want["runs"])
    assert int(got.status.item()) == want["status"]
    return want


def tables(old, page, width, g):
    """A block table whose pages so far are given out, and the free list."""
    have = [-(-max(int(o), 0) // page) for o in old]
    pool = g.permutation(sum(have) + 4 * len(old) * 40 + 8)
    table, at = np.full((len(old), width), -1, np.int32), 0
    for i, h in enumerate(have):
        h = min(h, width)
        table[i, :h] = pool[at:at + h]
        at += h
    return table, pool[at:].astype(np.int32)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("reqs,most_old,most_new,seed", [(1, 1, 1, 0), (1, 700, 2049, 1), (3, 600, 300, 2), (64, 500, 1, 3),
                                                         (257, 300, 40, 4), (1000, 64, 3, 5)])
def test_plan(uz, page, reqs, most_old, most_new, seed):
    g = np.random.default_rng(100 + seed)
    old, new = g.integers(0, most_old + 1, reqs), g.integers(0, most_new + 1, reqs)
    if reqs == 64:
        new[:] = 1
    table, free = tables(old, page, int((old + new).max()) // page + 2, g)
    need = int((-(-(old + new) // page) + old // -page).sum())
    check_plan(uz, old, new, free[:need], table, page, int(new.sum()))
    check_plan(uz, old, new, free[:need + 3], table, page, int(new.sum()) + 1031)


def test_plan_most_requests(uz):
    g = np.random.default_rng(7)
    n = uz.KV_MAX_REQUESTS
    old, new = g.integers(0, 100, n), g.integers(0, 30, n)
    table, free = tables(old, 16, 9, g)
    check_plan(uz, old, new, free, table, 16, int(new.sum()))


def test_plan_refuses_requests(uz):
    g = np.random.default_rng(8)
    old, new = [20, 16, 5, 40, 0, 3], [12, 17, 3, 33, 0, 1]
    table, free = tables(old, 16, 8, g)
    for pages in range(6):                                                # the list ends at each of them
        check_plan(uz, old, new, free[:pages], table, 16, sum(new))
    for rows in (0, 11, 12, 30, sum(new) - 1):                            # rows too few
        check_plan(uz, old, new, free, table, 16, rows)
    check_plan(uz, old, new, free, table[:, :3], 16, sum(new))            # a table too narrow
    check_plan(uz, [5, -1, 7, 9], [1, 2, -3, 4], free, np.zeros((4, 2), np.int32), 16, 40)
    check_plan(uz, [2 ** 31 - 1, 1], [1, 1], free, np.zeros((2, 2), np.int32), 16, 2)
    bad = [0, 0], [17, 3], np.array([-1, 3, 4], np.int32), np.full((2, 2), -1, np.int32)
    check_plan(uz, *bad, 16, 20)                                          # a page that is none: its rows have no slot
    p = uz.kv_plan(ints([0]), ints([16]), ints([]), ints([[-1]]), 16, 16)
    assert int(p.status.item()) == uz.ENOSPC
    with pytest.raises(uz.UzipError):
        uz.kv_plan(ints([0]), ints([16]), ints([]), ints([[-1]]), 16, 16, check=True)


def test_plan_of_nothing(uz):
    check_plan(uz, [], [], [1, 2], np.zeros((0, 3), np.int32), 16, 5)
    check_plan(uz, [], [], [], np.zeros((0, 3), np.int32), 16, 0)
    check_plan(uz, [4, 0], [0, 0], [], np.zeros((2, 1), np.int32), 16, 0)


# ------------------------------------------------------------------ a cache and its oracle side by side
class Side:
    def __init__(self, uz, pages, heads, page, dim, fmt, g):
        self.page, self.dim, self.fmt = page, dim, fmt
        # what unwritten pages hold: any bytes, NaN codes among them
        self.k = g.integers(0, 256, (pages, heads, page, dim), dtype=np.uint8)
        self.v = g.integers(0, 256, (pages, heads, page, dim), dtype=np.uint8)
        self.k_exp = g.integers(0, 256, (pages, heads), dtype=np.uint8)
        self.v_exp = g.integers(0, 256, (pages, heads), dtype=np.uint8)
        self.cache = uz.KVCache(dev(self.k), dev(self.k_exp), dev(self.v.transpose(0, 1, 3, 2)), dev(self.v_exp), fmt)

    def store(self, k, v, slots, runs):
        ref.store(self.k, self.k_exp, k, slots, runs, self.page, self.fmt)
        ref.store(self.v, self.v_exp, v, slots, runs, self.page, self.fmt)

    def check(self):
        torch.cuda.synchronize()
        assert np.array_equal(self.cache.k_exp.cpu().numpy(), self.k_exp)
        assert np.array_equal(self.cache.v_exp.cpu().numpy(), self.v_exp)
        assert np.array_equal(self.cache.k.cpu().numpy(), self.k)
        assert np.array_equal(self.cache.v.cpu().numpy().transpose(0, 1, 3, 2), self.v)


def rows_of(shape, kind, g, scale=1.0, fused=0, odd=False):
    """Values of a type, contiguous, or a slice of a wider array (fused: heads beside them; odd: at odd strides)."""
    x = torch.from_numpy(g.standard_normal(shape).astype(np.float32) * scale).to(TYPES[kind])
    rows, heads, dim = shape
    if odd:
        wide = torch.zeros(rows, heads, dim + 3, dtype=TYPES[kind], device="cuda")
        wide[:, :, 1:dim + 1] = x.cuda()
        return x, wide[:, :, 1:dim + 1]
    if fused:
        wide = torch.zeros(rows, heads + fused, dim, dtype=TYPES[kind], device="cuda")
        wide[:, 1:heads + 1] = x.cuda()
        return x, wide[:, 1:heads + 1]
    return x, x.cuda()


def grow(uz, side, old, new, table, free, kind, g, scale=1.0, fused=0, odd=False, edit=None):
    """One step through plan and store on both sides; returns the lengths after it and the plan."""
    rows = int(np.sum(new))
    want = ref.plan(old, new, free, table, side.page, rows)
    t = ints(table)
    plan = uz.kv_plan(ints(old), ints(new), ints(free), t, side.page, rows)
    heads = side.k.shape[1]
    k, kd = rows_of((rows, heads, side.dim), kind, g, scale, fused, odd)
    v, vd = rows_of((rows, heads, side.dim), kind, g, 3 * scale, fused, odd)
    if edit is not None:
        edit(k, kd)
        edit(v, vd)
    uz.kv_store(side.cache, kd, vd, plan.slots, plan.runs, plan.counts)
    with np.errstate(invalid="ignore"):
        side.store(np_of(k), np_of(v), want["slots"], want["runs"])
    return want["lens"], want, t


STORES = [  # page, dim, heads, kind, fmt, old, new, fused, odd
    (16, 64, 1, "bf16", "e4m3fn", [0], [1], 0, False),
    (64, 128, 2, "bf16", "e4m3fn", [0, 3, 64, 63], [64, 5, 1, 2], 3, False),
    (16, 96, 3, "fp16", "e5m2", [5, 0, 17], [40, 17, 15], 0, False),
    (256, 256, 1, "fp32", "e4m3fn", [1, 255], [300, 2], 2, False),
    (32, 192, 2, "fp32", "e5m2", [7, 31, 32], [1, 1, 1], 0, True),
    (128, 64, 2, "fp16", "e4m3fn", [100, 1], [60, 128], 0, True),
    (256, 64, 1, "bf16", "e5m2", [13], [511], 0, True),
    (16, 128, 4, "fp32", "e4m3fn", [15, 16, 1], [3, 33, 0], 1, False),
]


@pytest.mark.parametrize("case", STORES, ids=str)
def test_store(uz, case):
    page, dim, heads, kind, fmt, old, new, fused, odd = case
    say("store", case)
    g = np.random.default_rng(11)
    side = Side(uz, 40, heads, page, dim, fmt, g)
    free = g.permutation(40).astype(np.int32)
    table = np.full((len(old), 40), -1, np.int32)
    lens, want, _ = grow(uz, side, [0] * len(old), old, table, free, kind, g, fused=fused, odd=odd)   # what was there before
    side.check()
    free = free[want["counts"][0]:]
    for scale in (1.0, 40.0, 0.01):                                       # the second step's scales grow, the third's do not
        lens, want, _ = grow(uz, side, lens, new, want["table"], free, kind, g, scale, fused, odd)
        free = free[want["counts"][0]:]
        side.check()


@pytest.mark.parametrize("fmt", ["e4m3fn", "e5m2"])
@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
def test_store_of_special_values(uz, fmt, kind):
    say("special", fmt, kind)
    g = np.random.default_rng(12)
    side = Side(uz, 16, 2, 16, 64, fmt, g)
    big = float(torch.finfo(TYPES[kind]).max)
    tiny = float(torch.finfo(TYPES[kind]).smallest_normal) / 4
    top = ref.FORMATS[fmt][2]

    def edit(x, d):
        for t in (x, d):
            t[0] = 0.0                                                    # alone in its page: the least exponent
            t[1, 0, :4] = torch.tensor([float("nan"), float("inf"), -float("inf"), -0.0])
            t[2] = float("nan")
            t[3] = -float("inf")
            t[4] = tiny
            t[5, 0] = big
            t[6, 0] = -big
            t[7, 1] = min(top, big)                                       # just within the range, just past it
            t[8, 1] = min(top, big) * 1.01 if kind != "fp16" else 60000.0
            t[9:11] = 0.0
    free = np.arange(16, dtype=np.int32)
    table = np.full((12, 2), -1, np.int32)
    lens, want, _ = grow(uz, side, [0] * 12, [1] * 12, table, free, kind, g, edit=edit)
    side.check()
    grow(uz, side, lens, [1] * 12, want["table"], free[12:], kind, g, edit=edit)
    side.check()


def test_store_skips_what_has_no_place(uz):
    g = np.random.default_rng(13)
    side = Side(uz, 4, 2, 16, 64, "e4m3fn", g)
    for mine, its in ((side.k_exp, side.cache.k_exp), (side.v_exp, side.cache.v_exp)):
        mine[:] = 110                                                     # exponents that store can have written
        its.fill_(110)
    k, kd = rows_of((8, 2, 64), "bf16", g)
    slots = np.array([-1, -1, 64, 65, 16 * 3 + 14, 16 * 3 + 15, 2 ** 40, 5], np.int64)
    # no place; past the pool; three rows where two fit; rows that are not there; an empty run; the last row
    runs = [(0, 2), (2, 2), (4, 3), (-1, 3), (9, 1), (6, 1), (3, 0), (7, 4)]
    side.store(np_of(k), np_of(k), slots, [(4, 2), (7, 1)])
    uz.kv_store(side.cache, kd, kd, dev(slots), ints(runs), ints([0, len(runs)]))
    side.check()
    uz.kv_store(side.cache, kd, kd, dev(slots), ints(runs), ints([0, 0]))
    uz.kv_store(side.cache, kd, kd, dev(slots), ints(runs), ints([0, -5]))
    side.check()
    uz.kv_store(side.cache, kd[:0], kd[:0], dev(slots), ints(runs), ints([0, 0]))
    side.check()


# ------------------------------------------------------------------ attention
def run_attend(uz, side, q, table, lens, q_start, max_new, scale, window=0, out=None, lse=None, ws=None):
    return uz.kv_attend(q, side.cache, table, lens, q_start, max_new, scale=scale, window=window, out=out, lse=lse, ws=ws)


def check_attend(got, want, kind, dim, tokens):
    out, lse = got
    torch.cuda.synchronize()
    out, lse = np_of(out), lse.cpu().numpy().astype(np.float64)
    score = dim * 2.0 ** -24 * want["size"] + 2.0 ** -22 * want["size"] + 2.0 ** -21
    eps = 2 * (score + tokens * 2.0 ** -24)
    tol = U_OUT[kind] * np.abs(want["out"]) + (U_P[kind] + eps)[..., None] * want["spread"]
    tol += {"bf16": 2.0 ** -130, "fp16": 2.0 ** -25, "fp32": 2.0 ** -130}[kind]
    bad = ~(np.abs(out - want["out"]) <= tol)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:4].tolist(), (np.abs(out - want["out"]) / tol).max())
    empty = np.isneginf(want["lse"])
    assert np.array_equal(empty, np.isneginf(lse))
    with np.errstate(invalid="ignore"):
        assert (np.abs(lse - want["lse"])[~empty] <= (eps + 2.0 ** -22 * np.abs(want["lse"]))[~empty]).all()


def attend_case(uz, page, dim, kv, group, kind, fmt, ctx, new, window=0, fused=0, odd=False, scale=None, seed=21, pad=0,
                holes=False, wrong_max=None):
    g = np.random.default_rng(seed)
    total = [c + n for c, n in zip(ctx, new)]
    pages = sum(-(-t // page) for t in total) + 3
    side = Side(uz, pages, kv, page, dim, fmt, g)
    free = g.permutation(pages).astype(np.int32)
    table = np.full((len(ctx), max(-(-t // page) for t in total) + 1), -1, np.int32)
    _, want, _ = grow(uz, side, [0] * len(ctx), total, table, free, kind, g)
    table = want["table"]
    if holes:                                                             # pages that are none
        for i in range(len(ctx)):
            table[i, g.integers(0, table.shape[1])] = g.choice([-1, pages, 2 ** 31 - 1, -2 ** 31])
    rows = sum(new) + pad
    q, qd = rows_of((rows, kv * group, dim), kind, g, 2.0, fused, odd)
    scale = dim ** -0.5 if scale is None else scale
    q_start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    lens = np.array(total, np.int32)
    expect = ref.attend(np_of(q), side.k, side.k_exp, side.v, side.v_exp, fmt, table, lens, q_start, page, scale, window)
    out = None
    if odd:
        out = torch.full((rows, kv * group, dim + 3), 7.0, dtype=TYPES[kind], device="cuda")[:, :, 1:dim + 1]
    most = max(new) if wrong_max is None else wrong_max
    got = run_attend(uz, side, qd, ints(table), ints(lens), ints(q_start), most, scale, window, out)
    check_attend(got, expect, kind, dim, max(total) if total else 1)
    return side, qd, table, lens, q_start, scale, expect, got


ATTENDS = [  # page, dim, kv, group, kind, fmt, ctx, new, more
    (16, 64, 1, 1, "bf16", "e4m3fn", [0], [1], {}),
    (16, 64, 2, 7, "fp16", "e4m3fn", [37], [1], {}),
    (64, 128, 2, 4, "bf16", "e4m3fn", [0, 1, 63, 64, 65, 500], [1, 1, 1, 1, 1, 1], dict(fused=3)),
    (32, 128, 1, 8, "fp32", "e5m2", [15, 16, 17, 130, 1021], [1] * 5, {}),
    (128, 96, 3, 1, "bf16", "e5m2", [127, 128, 129, 700], [1, 2, 3, 4], {}),
    (256, 192, 1, 3, "fp16", "e5m2", [255, 256, 300], [5, 1, 7], dict(odd=True)),
    (16, 256, 2, 2, "fp32", "e4m3fn", [33, 400, 0], [5, 5, 5], dict(window=40)),
    (64, 256, 1, 8, "bf16", "e4m3fn", [700, 3], [3, 1], dict(window=1)),
    (64, 128, 1, 16, "fp16", "e4m3fn", [300], [1], {}),
    (64, 128, 1, 17, "bf16", "e4m3fn", [300], [1], dict(odd=True)),
    (64, 64, 1, 33, "bf16", "e4m3fn", [129], [2], {}),
    (64, 128, 2, 4, "bf16", "e4m3fn", [0], [200], {}),                    # prompts
    (16, 64, 2, 7, "fp16", "e4m3fn", [70, 0], [129, 61], dict(fused=4)),
    (128, 128, 1, 8, "bf16", "e5m2", [300, 5], [33, 100], dict(window=77)),
    (32, 96, 3, 1, "bf16", "e4m3fn", [5, 90, 31], [1, 140, 1], {}),       # mixed
    (256, 256, 1, 2, "fp16", "e4m3fn", [100], [130], dict(odd=True)),
    (32, 192, 1, 1, "bf16", "e4m3fn", [64], [257], {}),
    (64, 128, 1, 2, "fp32", "e4m3fn", [40, 0], [100, 90], {}),
    (16, 64, 1, 1, "bf16", "e4m3fn", [0, 0, 10], [1, 300, 0], {}),
]


@pytest.mark.parametrize("case", ATTENDS, ids=str)
def test_attend(uz, case):
    *args, more = case
    say("attend", case)
    attend_case(uz, *args, **more)


def test_attend_many_requests(uz):
    """More requests than a workgroup has threads, single tokens and pieces of prompts among them."""
    say("many requests")
    g = np.random.default_rng(81)
    n = 700
    ctx, new = g.integers(0, 60, n), np.where(g.random(n) < 0.03, 40, g.integers(0, 3, n))
    attend_case(uz, 16, 64, 1, 2, "bf16", "e4m3fn", ctx.tolist(), new.tolist())
    attend_case(uz, 32, 64, 1, 3, "fp16", "e5m2", ctx.tolist(), np.minimum(new, 2).tolist(), window=19)


@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows", [15, 17, 31, 33, 63, 65, 130])
def test_attend_on_both_sides_of_the_kernels_lines(uz, dim, kind, rows):
    """Lists of 16 rows, and the ends of blocks of 16, 32 and 128."""
    attend_case(uz, 64, dim, 1, 1, kind, "e4m3fn", [700, 3], [rows, 1], fused=1)


@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_attend_where_the_kernel_for_many_rows_begins(uz, dim, kind):
    """Lists of 96 or 160 rows, by dim, and the next; blocks of 128 and what is left of them."""
    for rows in (95, 96, 97, 127, 128, 129, 160, 161, 256, 257):
        attend_case(uz, 64, dim, 1, 1, kind, "e4m3fn", [300, 3], [rows, 2], seed=22)
    attend_case(uz, 16, dim, 2, 5, kind, "e5m2", [700, 0, 40, 5], [20, 30, 26, 19], seed=23, window=333)


@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
def test_attend_lists_of_17_to_32_rows_for_every_unit(uz, dim, kind):
    """Requests times heads past the compute units: blocks of 32 rows where there are such; one long list is split."""
    g = np.random.default_rng(24)
    ctx, new = g.integers(0, 90, 90), g.integers(0, 9, 90)
    ctx[7], new[7], new[8] = 3000, 8, 8
    attend_case(uz, 32, dim, 3, 4, kind, "e4m3fn", ctx.tolist(), new.tolist(), seed=25)
    attend_case(uz, 16, dim, 3, 6, kind, "e5m2", ctx.tolist(), np.minimum(new, 5).tolist(), seed=26, window=50, holes=True)


@pytest.mark.parametrize("dim,kind", [(64, "bf16"), (64, "fp32"), (96, "fp16")])
def test_attend_long_lists_for_half_the_units(uz, dim, kind):
    """136 blocks of long requests, and of less long ones: where the length of a piece changes its rule."""
    attend_case(uz, 128, dim, 8, 1, kind, "e4m3fn", [4200] * 17, [1] * 17, seed=27)
    attend_case(uz, 128, dim, 8, 1, kind, "e4m3fn", [4200] * 16 + [3], [2] * 17, seed=28, window=3000)


@pytest.mark.parametrize("fmt", ["e4m3fn", "e5m2"])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_attend_nan_and_infinity_in_blocks_of_32_rows(uz, fmt, kind):
    g = np.random.default_rng(74)
    n, total, new, page, dim = 130, 40, 9, 16, 64
    side = Side(uz, 3 * n, 2, page, dim, fmt, g)

    def edit(x, d):
        for t in (x, d):
            if edit.values:
                for i in range(0, n, 3):
                    for tok, ch, v in ((33, 3, "nan"), (35, 3, "inf"), (36, 5, "-inf"), (38, 6, "inf"), (39, 6, "-inf"), (2, 9, "inf")):
                        t[i * total + tok, i % 2, ch] = float(v)
        edit.values = True
    edit.values = False
    _, want, _ = grow(uz, side, [0] * n, [total] * n, np.full((n, 4), -1, np.int32), np.arange(3 * n, dtype=np.int32), kind, g, edit=edit)
    q, qd = rows_of((n * new, 4, dim), kind, g)
    q_start = np.arange(n + 1, dtype=np.int32) * new
    for window in (0, 12):
        with np.errstate(invalid="ignore"):
            expect = ref.attend(np_of(q), side.k, side.k_exp, side.v, side.v_exp, fmt, want["table"], [total] * n, q_start, page, 0.1, window)
        out, lse = run_attend(uz, side, qd, ints(want["table"]), ints([total] * n), ints(q_start), new, 0.1, window)
        got, fine = np_of(out), np.isfinite(expect["out"])
        assert not fine.all() and fine.any()
        assert np.array_equal(got[~fine], expect["out"][~fine], equal_nan=True)
        assert np.isfinite(got[fine]).all()
        clean = {k: np.where(fine, v, 0.0) if k in ("out", "spread") else v for k, v in expect.items()}
        check_attend((torch.from_numpy(np.where(fine, got, 0.0)), lse), clean, kind, dim, total)


@pytest.mark.parametrize("kind,dim,ctx", [("bf16", 128, 5000), ("fp16", 64, 4097), ("fp32", 96, 3333)])
def test_attend_long_contexts_are_split_and_joined(uz, kind, dim, ctx):
    say("long", kind, dim, ctx)
    attend_case(uz, 64, dim, 1, 2, kind, "e4m3fn", [ctx, 10], [1, 1])
    attend_case(uz, 16, dim, 2, 1, kind, "e4m3fn", [ctx], [40])


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
def test_attend_rows_without_tokens(uz, kind):
    """Rows of empty requests, rows before the first place, rows of no request, pages that are none."""
    say("empty rows", kind)
    attend_case(uz, 16, 64, 2, 3, kind, "e4m3fn", [20, 0, 5], [1, 2, 1], pad=9)
    attend_case(uz, 16, 64, 2, 3, kind, "e4m3fn", [90, 40, 260], [1, 50, 3], holes=True)
    g = np.random.default_rng(31)
    side = Side(uz, 8, 1, 16, 64, "e4m3fn", g)
    free = np.arange(8, dtype=np.int32)
    _, want, _ = grow(uz, side, [0, 0], [64, 30], np.full((2, 4), -1, np.int32), free, kind, g)
    q, qd = rows_of((90, 2, 64), kind, g)
    q_start = np.array([0, 40, 85], np.int32)                             # more rows than tokens, some rows of no request
    for lens in ([20, 30], [0, 30], [-7, 0], [2 ** 31 - 1, 17]):              # a length past the table counts as 64
        expect = ref.attend(np_of(q), side.k, side.k_exp, side.v, side.v_exp, "e4m3fn", want["table"], lens, q_start, 16, 0.2)
        assert np.isneginf(expect["lse"]).any()
        got = run_attend(uz, side, qd, ints(want["table"]), ints(lens), ints(q_start), 45, 0.2)
        check_attend(got, expect, kind, 64, 64)
        assert (got[0][85:] == 0).all() and torch.isneginf(got[1][85:]).all()


def test_attend_of_no_requests(uz):
    g = np.random.default_rng(32)
    side = Side(uz, 2, 1, 16, 64, "e4m3fn", g)
    q, qd = rows_of((5, 2, 64), "bf16", g)
    out, lse = run_attend(uz, side, qd, ints(np.zeros((0, 1))), ints([]), ints([0]), 1, 1.0)
    assert (out == 0).all() and torch.isneginf(lse).all()
    out, _ = run_attend(uz, side, qd[:0], ints(np.zeros((0, 1))), ints([]), ints([0]), 1, 1.0)
    assert out.shape == (0, 2, 64)


@pytest.mark.parametrize("most", [0, 1, 7, 1 << 20])
def test_attend_whatever_max_new_says(uz, most):
    say("max_new", most)
    attend_case(uz, 32, 64, 2, 4, "bf16", "e4m3fn", [100, 3, 500], [90, 1, 4], wrong_max=most)


def test_attend_pages_of_very_different_scales(uz):
    """Pages whose scales lie far apart: no probability may be lost to a type's range."""
    say("scales")
    for kind in ("bf16", "fp16", "fp32"):
        g = np.random.default_rng(33)
        side = Side(uz, 8, 1, 16, 64, "e4m3fn", g)
        _, want, _ = grow(uz, side, [0], [64], np.full((1, 4), -1, np.int32), np.arange(4, dtype=np.int32), kind, g)
        for i, e in enumerate((30, 120, 200, 127)):
            side.v_exp[i] = e
        side.v_exp[2] = 130 if kind == "fp16" else 200                    # fp16 outputs have to stay finite
        side.cache.v_exp.copy_(dev(side.v_exp))
        q, qd = rows_of((1, 1, 64), kind, g)
        for page in range(4):                                             # nearly all weight on one page
            kk = ref.decode(side.k[want["table"][0, page], 0], "e4m3fn", side.k_exp[want["table"][0, page], 0])
            q[0, 0] = torch.from_numpy(kk[3] * 3).to(TYPES[kind])
            qd.copy_(q.cuda())
            expect = ref.attend(np_of(q), side.k, side.k_exp, side.v, side.v_exp, "e4m3fn", want["table"], [64], [0, 1], 16, 1.0)
            got = run_attend(uz, side, qd, ints(want["table"]), ints([64]), ints([0, 1]), 1, 1.0)
            check_attend(got, expect, kind, 64, 64)


def test_attend_large_scores(uz):
    """Scores of thousands: the running maximum keeps every exponential in range."""
    for kind in ("bf16", "fp16", "fp32"):
        attend_case(uz, 16, 64, 1, 2, kind, "e4m3fn", [100, 700], [1, 70], scale=50.0)
        attend_case(uz, 16, 64, 1, 2, kind, "e4m3fn", [100], [1], scale=-1.0)
        attend_case(uz, 16, 64, 1, 2, kind, "e4m3fn", [100], [1], scale=0.0)


@pytest.mark.parametrize("fmt", ["e4m3fn", "e5m2"])
@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("new,window", [([6, 1], 0), ([6, 3], 9), ([30, 24], 0), ([31, 2], 9), ([100, 70], 0), ([90, 1], 33)])
def test_attend_nan_and_infinity_reach_only_rows_that_see_them(uz, fmt, kind, new, window):
    say("nan", fmt, kind, new, window)
    g = np.random.default_rng(71)
    page, dim, kv, group = 16, 64, 2, 2
    side = Side(uz, 24, kv, page, dim, fmt, g)
    total = [130, 75]

    def edit(x, d):
        for t in (x, d):
            if x.stride(0) and edit.values:                               # values only: a key's NaN is another test
                for tok, ch, v in [(124, 3, "nan"), (127, 3, "inf"), (126, 5, "inf"), (128, 6, "-inf"), (129, 6, "inf"), (60, 9, "nan"),
                                   (40, 11, "inf"), (130 + 72, 1, "nan"), (130 + 20, 2, "-inf")]:
                    t[tok, 1, ch] = float(v)
        edit.values = True                                                # grow edits keys first
    edit.values = False
    _, want, _ = grow(uz, side, [0, 0], total, np.full((2, 12), -1, np.int32), np.arange(24, dtype=np.int32), kind, g, edit=edit)
    rows = sum(new)
    q, qd = rows_of((rows, kv * group, dim), kind, g)
    q_start = np.array([0, new[0], rows], np.int32)
    with np.errstate(invalid="ignore"):
        expect = ref.attend(np_of(q), side.k, side.k_exp, side.v, side.v_exp, fmt, want["table"], total, q_start, page, 0.1, window)
    out, lse = run_attend(uz, side, qd, ints(want["table"]), ints(total), ints(q_start), max(new), 0.1, window)
    got, fine = np_of(out), np.isfinite(expect["out"])
    assert not fine.all() and fine.any()
    assert np.array_equal(got[~fine], expect["out"][~fine], equal_nan=True)
    assert np.isfinite(got[fine]).all()
    clean = {k: np.where(fine, v, 0.0) if k in ("out", "spread") else v for k, v in expect.items()}
    check_attend((torch.from_numpy(np.where(fine, got, 0.0)), lse), clean, kind, dim, 130)


@pytest.mark.parametrize("fmt", ["e4m3fn", "e5m2"])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("new", [3, 20, 50, 90])
def test_attend_nan_beside_a_page_that_is_none(uz, fmt, kind, new):
    """A NaN that all rows see, in a step of which another page is missing, reaches all rows."""
    g = np.random.default_rng(73)
    side = Side(uz, 24, 1, 16, 64, fmt, g)

    def edit(x, d):
        for t in (x, d):
            if edit.values:
                t[20, 0, 5] = float("nan")
                t[21, 0, 6] = float("inf")
        edit.values = True
    edit.values = False
    _, want, _ = grow(uz, side, [0], [300], np.full((1, 20), -1, np.int32), np.arange(24, dtype=np.int32), kind, g, edit=edit)
    table = want["table"]
    table[0, 2] = -1
    q, qd = rows_of((new, 2, 64), kind, g)
    with np.errstate(invalid="ignore"):
        expect = ref.attend(np_of(q), side.k, side.k_exp, side.v, side.v_exp, fmt, table, [300], [0, new], 16, 0.1)
    out, _ = run_attend(uz, side, qd, ints(table), ints([300]), ints([0, new]), new, 0.1)
    got, fine = np_of(out), np.isfinite(expect["out"])
    assert not fine[:, :, 5].any() and not fine[:, :, 6].any() and fine[:, :, :5].all()
    assert np.array_equal(got[~fine], expect["out"][~fine], equal_nan=True) and np.isfinite(got[fine]).all()


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("new", [[5], [100]])
def test_attend_nan_keys_reach_only_rows_that_see_them(uz, kind, new):
    g = np.random.default_rng(72)
    side = Side(uz, 10, 1, 16, 64, "e4m3fn", g)

    def edit(x, d):
        for t in (x, d):
            t[117, 0, 7] = float("nan")
    _, want, _ = grow(uz, side, [0], [120], np.full((1, 8), -1, np.int32), np.arange(10, dtype=np.int32), kind, g, edit=edit)
    q, qd = rows_of((new[0], 2, 64), kind, g)
    out, lse = run_attend(uz, side, qd, ints(want["table"]), ints([120]), ints([0, new[0]]), new[0], 0.1)
    torch.cuda.synchronize()
    first = 117 - (120 - new[0])
    assert torch.isfinite(out[:first]).all() and torch.isfinite(lse[:first]).all()
    assert torch.isnan(out[first:]).all() and torch.isnan(lse[first:]).all()


def test_attend_repeats_its_bits(uz):
    """The same call gives the same bits, on a workspace that holds anything, on another stream, without lse."""
    for new in ([1, 1, 1], [3, 150, 1]):
        side, qd, table, lens, q_start, scale, expect, got = attend_case(uz, 32, 128, 2, 4, "bf16", "e4m3fn", [3000, 40, 900], new)
        args = ints(table), ints(lens), ints(q_start), max(new), scale
        ws = uz.kv_attend_workspace(qd, side.cache, 3, max(new))
        for fill in (0, 255):
            ws.fill_(fill)
            out, lse = run_attend(uz, side, qd, *args, ws=ws)
            assert torch.equal(out, got[0]) and torch.equal(lse, got[1])
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        out, lse = uz.kv_attend(qd, side.cache, *args[:4], scale=scale, stream=s, ws=ws, out=torch.zeros_like(out),
                                lse=torch.zeros_like(lse))
        s.synchronize()
        assert torch.equal(out, got[0]) and torch.equal(lse, got[1])


def test_cache_past_32_bits(uz):
    """A pool whose bytes pass 2^32: the last pages are found."""
    say("large pool")
    pages, heads, page, dim = 33000, 16, 64, 128                          # 4.3 GB each of keys and values
    cache = uz.KVCache.empty(pages, heads, dim, page)
    g = np.random.default_rng(41)
    free = np.array([pages - 1, 0, pages - 2], np.int32)
    plan = uz.kv_plan(ints([0, 0]), ints([100, 30]), ints(free), ints(np.full((2, 2), -1)), page, 130)
    t = ints([[pages - 1, 0], [pages - 2, -1]])
    k, kd = rows_of((130, heads, dim), "bf16", g)
    v, vd = rows_of((130, heads, dim), "bf16", g)
    uz.kv_store(cache, kd, vd, plan.slots, plan.runs, plan.counts)
    small = Side(uz, 3, heads, page, dim, "e4m3fn", g)
    lens, starts = [100, 30], [0, 100, 130]
    slots = np.concatenate([np.arange(100), np.arange(128, 158)])
    small.store(np_of(k), np_of(v), slots, [(0, 64), (64, 36), (100, 30)])
    idx = torch.tensor([pages - 1, 0, pages - 2], device="cuda")
    assert np.array_equal(cache.k[idx].cpu().numpy()[0], small.k[0]) and \
        np.array_equal(cache.v[idx].cpu().numpy().transpose(0, 1, 3, 2)[0], small.v[0])
    q, qd = rows_of((130, heads, dim), "bf16", g)
    expect = ref.attend(np_of(q), small.k, small.k_exp, small.v, small.v_exp, "e4m3fn", np.array([[0, 1], [2, -1]]), lens, starts,
                        page, dim ** -0.5)
    got = uz.kv_attend(qd, cache, t, ints(lens), ints(starts), 100)
    check_attend(got, expect, "bf16", dim, 100)
    del cache
    torch.cuda.empty_cache()


def test_a_step_in_a_graph(uz):
    """plan, store and attend captured once and replayed with other lengths and values."""
    g = np.random.default_rng(51)
    reqs, heads, group, page, dim, width = 3, 2, 2, 16, 64, 20
    side = Side(uz, 70, heads, page, dim, "e4m3fn", g)
    eager = Side(uz, 70, heads, page, dim, "e4m3fn", np.random.default_rng(51))
    free = g.permutation(70).astype(np.int32)
    rows = reqs
    table = ints(np.full((reqs, width), -1))
    old, new, fr = ints([0, 0, 0]), ints([1, 1, 1]), ints(free)
    k, v = (torch.zeros(rows, heads, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros(rows, heads * group, dim, dtype=torch.bfloat16, device="cuda")
    plan = uz.kv_plan_buffers(reqs, rows, page)
    out, lse = torch.zeros_like(q), torch.zeros(rows, heads * group, device="cuda")
    ws = uz.kv_attend_workspace(q, side.cache, reqs, 1)

    def step(cache, o, s, w, st=None):
        uz.kv_plan(old, new, fr, table, page, rows, out=plan, stream=st)
        uz.kv_store(cache, k, v, plan.slots, plan.runs, plan.counts, stream=st)
        return uz.kv_attend(q, cache, table, plan.lens, plan.q_start, 1, out=o, lse=s, ws=w, stream=st)
    step(eager.cache, out, lse, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(side.cache, out, lse, ws)
    table.fill_(-1)
    at, used = np.array([0, 0, 0]), 0
    for turn in range(40):
        fr.copy_(ints(np.roll(free, -used)))
        n = np.array([1, 1, 0]) if turn % 3 == 2 else np.array([1, 1, 1])
        old.copy_(ints(at))
        new.copy_(ints(n))
        for t in (k, v, q):
            t.copy_(torch.from_numpy(g.standard_normal(t.shape).astype(np.float32)).to(t.dtype))
        before = table.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        after = table.clone()
        table.copy_(before)
        want = step(eager.cache, torch.zeros_like(out), torch.zeros_like(lse), None)
        torch.cuda.synchronize()
        assert torch.equal(after, table) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), turn
        assert torch.equal(side.cache.k_exp[after[0, 0]], eager.cache.k_exp[after[0, 0]])
        used += int(plan.counts[0])
        at = at + n


def test_refusals_of_the_wrappers(uz):
    g = np.random.default_rng(61)
    side = Side(uz, 2, 1, 16, 64, "e4m3fn", g)
    c = side.cache
    with pytest.raises(ValueError):
        uz.KVCache(c.k.cpu(), c.k_exp, c.v, c.v_exp)
    with pytest.raises(ValueError):
        uz.KVCache(c.k, c.k_exp, c.k, c.v_exp)
    with pytest.raises(ValueError):
        uz.KVCache(c.k, c.k_exp, c.v, c.v_exp, "bf16")
    with pytest.raises(ValueError):
        uz.KVCache(c.k[:, :, ::2], c.k_exp, c.v[..., ::2], c.v_exp)
    q = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    t, n, s = ints([[0]]), ints([2]), ints([0, 2])
    bad = [dict(q=q.double()), dict(q=q[:, :, ::2]), dict(q=q.cpu()), dict(lens=n.long()), dict(q_start=s[:1]), dict(table=t[0]),
           dict(window=-1), dict(out=q[:1]), dict(out=q.float()), dict(lse=torch.zeros(2, 2, dtype=torch.float16, device="cuda"))]
    for b in bad:
        a = {"q": q, "table": t, "lens": n, "q_start": s, **b}
        with pytest.raises(ValueError):
            uz.kv_attend(a["q"], c, a["table"], a["lens"], a["q_start"], 2, window=a.get("window", 0), out=a.get("out"),
                         lse=a.get("lse"))
    with pytest.raises(uz.UzipError) as e:
        uz.kv_attend(q, c, t, n, s, 2, ws=torch.zeros(1, dtype=torch.uint8, device="cuda"))
    assert e.value.status == uz.ENOSPC
    with pytest.raises(uz.UzipError):
        uz.kv_attend(torch.zeros(2, 0, 64, dtype=torch.bfloat16, device="cuda"), c, t, n, s, 2)
    plan = uz.kv_plan_buffers(1, 2, 16)
    with pytest.raises(ValueError):
        uz.kv_store(c, q, q, plan.slots, plan.runs, plan.counts)          # two heads into a cache of one
    with pytest.raises(ValueError):
        uz.kv_plan(n, n, n, t, 16, 100, out=plan)
    with pytest.raises(uz.UzipError):
        uz.kv_plan(n, n, n, t, 17, 2, out=None)


def test_handoff_example():
    """Plan, store, attend and the codec together: a cache handed over answers as the one that stayed, bit for bit."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "kv_handoff.py")
    spec = importlib.util.spec_from_file_location("kv_handoff", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    assert mod.main(prompts=(130, 1, 300), answer=70) == 0
