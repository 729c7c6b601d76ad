"""GPU: the paged 8-bit latent cache and both forms of its attention against oracle/latent.py in 64 bits.

Tolerance of an output: its own rounding (half an ulp); its weights, which enter the second product in terms of
four bits each, 8 bits for bf16 and 12 for fp16 (expanded form: as one number of the type, 8 and 11 bits), with the last
term's least step below that (`floor`, in units of the largest weight: 2^-17 and 2^-21; expanded fp16 2^-25); the 8-bit
matrix instruction, which drops what lies 2^-13 below the largest of eight products: for each of eight at most
that, 2^-10 of the sum of magnitudes; the scores, by their products' sums (width * 2^-24 of the sum of magnitudes), the
exponential (2^-22 of the score and 2^-21) and the token's exponent added to them (2^-23 of it), twice, in numerator
and sum; the row's sum (tokens * 2^-24).
"""
import numpy as np
import pytest
import torch

from oracle import kv as ref_kv
from oracle import latent as ref
from oracle import rotary as ref_rotary

from test_gpu_rotary import LEAST, TYPES, U_OUT, check as check_turned, dev, freq_of, ints, np_of, rows_of

pytestmark = pytest.mark.gpu

U_P = {"bf16": 2.0 ** -8 + 2.0 ** -10, "fp16": 2.0 ** -12 + 2.0 ** -10}
FLOOR = {"bf16": 2.0 ** -17, "fp16": 2.0 ** -21}
U_EXPANDED = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
FLOOR_EXPANDED = {"bf16": 0.0, "fp16": 2.0 ** -25}


def say(*a):
    print("[latent]", *a, flush=True)


@pytest.fixture(scope="module")
def uz():
    import paper_2604_17172_amd as m
    return m


def check_attend(got, want, kind, width, tokens, u_p, floor):
    out, lse = got
    torch.cuda.synchronize()
    out, lse = np_of(out), lse.cpu().numpy().astype(np.float64)
    shift = want.get("shift", 0.0)
    score = width * 2.0 ** -24 * want["size"] + 2.0 ** -22 * want["size"] + 2.0 ** -21 + 2.0 ** -23 * shift
    eps = 2 * (score + tokens * 2.0 ** -24)
    tol = U_OUT[kind] * np.abs(want["out"]) + (u_p + eps)[..., None] * want["spread"] + floor * want["floor"] + LEAST[kind]
    off = np.abs(out - want["out"])
    bad = ~(off <= tol)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:4].tolist(), np.nanmax(off / tol))
    empty = np.isneginf(want["lse"])
    assert np.array_equal(empty, np.isneginf(lse)) and (out[empty] == 0).all()
    with np.errstate(invalid="ignore"):
        far = np.abs(lse - want["lse"])[~empty]
    assert (far <= (eps + 2.0 ** -22 * np.abs(want["lse"]))[~empty]).all(), far.max()


class Side:
    """A cache on the GPU and its arrays on the host."""

    def __init__(self, uz, pages, page, latent, rot, fmt, g, spread=0):
        self.codes = (g.integers(0, 256, (pages, page, latent + rot)) & 0xBB).astype(np.uint8)  # no NaN, no infinity
        self.exps = g.integers(118 - spread, 124 + spread, (pages, page, 2)).astype(np.uint8)
        self.page, self.latent, self.rot, self.fmt = page, latent, rot, fmt
        self.cache = uz.LatentCache(dev(self.codes), dev(self.exps), rot, fmt)

    def refresh(self):
        self.cache.codes.copy_(dev(self.codes))
        self.cache.exps.copy_(dev(self.exps))


# ------------------------------------------------------------------ store
STORES = [  # page, latent, rot, heads, kind, fmt, old, new, interleaved, how
    (16, 512, 64, 0, "bf16", "e4m3fn", [0], [1], False, ""),
    (64, 512, 64, 16, "bf16", "e4m3fn", [0, 3, 64, 63], [64, 5, 1, 2], False, "fused"),
    (16, 256, 32, 3, "fp16", "e5m2", [5, 0, 17], [40, 17, 15], True, "odd"),
    (256, 256, 64, 1, "fp32", "e4m3fn", [1, 255], [300, 2], False, ""),
    (128, 512, 32, 7, "fp32", "e5m2", [7, 31, 32], [1, 1, 1], True, "odd"),
    (32, 256, 32, 128, "bf16", "e5m2", [9], [33], True, "fused"),
]


@pytest.mark.parametrize("case", STORES, ids=str)
def test_store(uz, case):
    page, latent, rot, heads, kind, fmt, old, new, interleaved, how = case
    say("store", case)
    g = np.random.default_rng(11)
    pages, freq = 40, freq_of(rot)
    side = Side(uz, pages, page, latent, rot, fmt, g)
    free = g.permutation(pages).astype(np.int32)
    table = np.full((len(old), 40), -1, np.int32)
    for i, o in enumerate(old):
        n = -(-o // page)
        table[i, :n], free = free[:n], free[n:]
    rows = int(np.sum(new)) + 2                                           # and two rows of no request
    plan = uz.kv_plan(ints(old), ints(new), ints(free), ints(table), page, rows)
    want = ref_kv.plan(old, new, free, table, page, rows)
    places = uz.kv_positions(plan.lens, plan.q_start, rows)
    c = rows_of((rows, 1, latent), kind, g, how, 3.0)[:, 0]
    k = rows_of((rows, 1, rot), kind, g, how, 0.3)[:, 0]
    c[0] *= 100
    c[-3] = 0                                                             # the least scale
    q = rows_of((rows, heads, rot), kind, g, how) if heads else None
    got = uz.latent_store(side.cache, c, k, places, dev(freq), plan.slots, q=q, interleaved=interleaved, magnitude=1.1)
    torch.cuda.synchronize()
    at = ref_rotary.positions(want["lens"], want["q_start"], rows)
    if q is None:
        assert got is None
    else:
        check_turned(got, q, at, freq, kind, interleaved=interleaved, magnitude=1.1)
    x = np_of(k)[:, None]
    turned, off = (f(x, at, freq, interleaved, 0, 1.1)[:, 0] for f in (ref_rotary.rotate, ref_rotary.error))
    ends = []
    for sign in (-1, 1):                                                  # the codes of the least and the largest it may be
        codes, exps = side.codes.copy(), side.exps.copy()
        ref.store(codes, exps, np_of(c), turned + sign * off, want["slots"], page, fmt)
        ends.append((codes, exps))
    codes, exps = side.cache.codes.cpu().numpy(), side.cache.exps.cpu().numpy()
    assert np.array_equal(exps[..., 0], ends[0][1][..., 0]) and np.array_equal(codes[..., :latent], ends[0][0][..., :latent])
    assert ((exps == ends[0][1]) | (exps == ends[1][1])).all()
    same = (exps == ends[0][1])[..., 1] & (exps == ends[1][1])[..., 1]
    ok = ((codes == ends[0][0]) | (codes == ends[1][0]))[..., latent:]
    assert ok[same].all() and (ends[0][0] != ends[1][0]).mean() < 1e-3


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("fmt", ["e4m3fn", "e5m2"])
def test_store_of_special_values(uz, fmt, kind):
    """NaN, infinities and the type's ends, and slots that are none; what is not stored to keeps its bytes."""
    g = np.random.default_rng(12)
    side = Side(uz, 3, 16, 256, 32, fmt, g)
    rows = 9
    c, k = rows_of((rows, 1, 256), kind, g)[:, 0], rows_of((rows, 1, 32), kind, g)[:, 0]
    top, least = torch.finfo(TYPES[kind]).max, torch.finfo(TYPES[kind]).smallest_normal
    c[0, 5], c[0, 6], c[0, 7] = float("nan"), float("inf"), float("-inf")
    c[1], c[2] = float("inf"), float("nan")
    c[3, 9], c[4, 0] = top, -top
    c[5] = least
    c[6], c[6, 3] = 0, least
    slots = torch.tensor([0, 5, 16, 17, 30, 47, 1, -1, 48], device="cuda")
    uz.latent_store(side.cache, c, k, ints(np.zeros(rows)), dev(freq_of(32)), slots)
    with np.errstate(invalid="ignore"):
        ref.store(side.codes, side.exps, np_of(c), np_of(k), slots.cpu().numpy(), 16, fmt)
    assert np.array_equal(side.cache.exps.cpu().numpy(), side.exps)
    assert np.array_equal(side.cache.codes.cpu().numpy(), side.codes)


# ------------------------------------------------------------------ absorbed form
def attend_case(uz, page, latent, rot, heads, kind, fmt, ctx, new, how="", scale=None, seed=21, pad=0, holes=False, most=None, spread=0,
                edit=None, q_scale=1.0):
    g = np.random.default_rng(seed)
    total = [c + n for c, n in zip(ctx, new)]
    pages = sum(-(-max(t, 0) // page) for t in total) + 3
    side = Side(uz, pages, page, latent, rot, fmt, g, spread)
    free = list(g.permutation(pages))
    table = np.full((len(ctx), max([-(-max(t, 0) // page) for t in total] + [0]) + 1), -1, np.int32)
    for i, t in enumerate(total):
        for j in range(-(-max(t, 0) // page)):
            table[i, j] = free.pop()
    if holes:                                                             # pages that are none
        for i in range(len(ctx)):
            table[i, g.integers(0, table.shape[1])] = g.choice([-1, pages, 2 ** 31 - 1, -2 ** 31])
    rows = sum(new) + pad
    q = rows_of((rows, heads, latent + rot), kind, g, how, q_scale)
    scale = 0.004 if scale is None else scale
    q_start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    lens = np.array(total, np.int32)
    if edit is not None:
        edit(side, table, q)
        side.refresh()
    with np.errstate(invalid="ignore", over="ignore"):
        want = ref.attend(np_of(q), side.codes, side.exps, latent, fmt, table, lens, q_start, page, scale)
    out = None
    if how == "odd":
        out = torch.full((rows, heads, latent + 3), 7.0, dtype=TYPES[kind], device="cuda")[:, :, 1:latent + 1]
    got = uz.latent_attend(q, side.cache, ints(table), ints(lens), ints(q_start), max(new) if most is None else most, scale, out=out)
    torch.cuda.synchronize()
    if edit is None:
        check_attend(got, want, kind, latent + rot, max(total + [1]), U_P[kind], FLOOR[kind])
    return side, q, table, lens, q_start, scale, want, got


ATTENDS = [  # page, latent, rot, heads, kind, fmt, ctx, new, more
    (16, 512, 64, 1, "bf16", "e4m3fn", [0], [1], {}),
    (16, 256, 32, 1, "fp16", "e5m2", [0], [1], {}),
    (16, 512, 64, 16, "bf16", "e4m3fn", [37], [1], {}),
    (64, 512, 64, 16, "fp16", "e4m3fn", [0, 1, 62, 63, 64, 126, 127, 128, 500], [1] * 9, {}),
    (32, 256, 64, 33, "bf16", "e5m2", [15, 16, 17, 130, 1021], [1] * 5, dict(how="fused")),
    (128, 512, 32, 64, "bf16", "e5m2", [127, 128, 129], [1, 2, 3], {}),
    (256, 256, 32, 128, "fp16", "e4m3fn", [255, 256, 300], [1, 1, 2], dict(how="odd")),
    (16, 512, 64, 5, "bf16", "e4m3fn", [100, 0, 3], [13, 70, 1], dict(how="odd")),
    (64, 256, 64, 3, "bf16", "e4m3fn", [0, 33], [150, 40], {}),
    (64, 512, 64, 2, "fp16", "e5m2", [11], [129], dict(how="fused")),
    (64, 512, 64, 31, "bf16", "e4m3fn", [190, 7], [1, 4], dict(pad=3)),
    (16, 256, 32, 8, "bf16", "e4m3fn", [70, 300, 5], [4, 9, 1], dict(holes=True)),
    (64, 512, 64, 16, "fp16", "e4m3fn", [400, 300], [1, 1], dict(holes=True)),
    (64, 256, 32, 16, "bf16", "e4m3fn", [200] * 3, [1, 8, 0], dict(spread=40)),
    (64, 512, 64, 16, "fp16", "e4m3fn", [200] * 3, [1, 8, 0], dict(spread=12)),
    (64, 512, 64, 16, "bf16", "e4m3fn", [100, 40], [2, 3], dict(scale=-0.01)),
    (64, 256, 32, 16, "fp16", "e5m2", [100, 40], [2, 3], dict(scale=0.0)),
    (16, 256, 32, 1, "bf16", "e4m3fn", [0, 0, 10], [1, 200, 0], {}),
]


@pytest.mark.parametrize("case", ATTENDS, ids=str)
def test_attend(uz, case):
    *args, more = case
    say("attend", case)
    *_, got = attend_case(uz, *args, **more)
    if more.get("how") == "odd":                                          # nothing beside the rows is written
        out = got[0]
        base = torch.as_strided(out, (*out.shape[:2], out.shape[2] + 3), out.stride(), out.storage_offset() - 1)
        assert (base[:, :, 0] == 7).all() and (base[:, :, -2:] == 7).all()


@pytest.mark.parametrize("latent", [256, 512])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("ctx,heads", [(5000, 16), (3333, 40), (4096, 128)])
def test_attend_long_contexts_are_split_and_joined(uz, kind, latent, ctx, heads):
    say("long", kind, latent, ctx, heads)
    attend_case(uz, 64, latent, 64, heads, kind, "e4m3fn", [ctx, 3, ctx // 2], [1, 1, 2])


def test_attend_many_requests(uz):
    g = np.random.default_rng(5)
    ctx = g.integers(0, 90, 300).tolist()
    attend_case(uz, 16, 256, 32, 2, "bf16", "e4m3fn", ctx, g.integers(0, 3, 300).tolist(), most=2)


@pytest.mark.parametrize("n", [15, 16, 17, 33, 48, 63, 64, 65, 130])
def test_attend_shares_of_so_many_requests(uz, n):
    """The work before a request is summed over lanes, several requests to one from 64 on."""
    g = np.random.default_rng(n)
    ctx = (g.integers(0, 2, n) * g.integers(0, 1500, n)).tolist()
    new = g.integers(0, 3, n).tolist()
    new[n // 2] = 40
    attend_case(uz, 16, 256, 32, 5, "bf16", "e4m3fn", ctx, new)


@pytest.mark.parametrize("most", [0, 1, 7, 1 << 20])
def test_attend_whatever_max_new_says(uz, most):
    attend_case(uz, 64, 512, 64, 12, "bf16", "e4m3fn", [100, 5, 700], [5, 9, 1], most=most)


def test_attend_large_scores(uz):
    """Scores in the thousands: one token takes all the weight."""
    attend_case(uz, 64, 512, 64, 16, "bf16", "e4m3fn", [500], [3], scale=3.0)
    attend_case(uz, 64, 256, 64, 16, "fp16", "e4m3fn", [500], [3], scale=2.0)


def test_attend_rows_without_tokens(uz):
    """Requests of length 0, places before the first token, rows of no request."""
    g = np.random.default_rng(6)
    side = Side(uz, 5, 16, 256, 32, "e4m3fn", g)
    table, lens, q_start = np.array([[0, 1], [2, -1], [3, -1], [-1, -1]], np.int32), np.array([0, 3, 16, 5], np.int32), np.array([0, 2, 8, 9, 10], np.int32)
    q = rows_of((13, 3, 288), "bf16", g)
    want = ref.attend(np_of(q), side.codes, side.exps, 256, "e4m3fn", table, lens, q_start, 16, 0.01)
    got = uz.latent_attend(q, side.cache, ints(table), ints(lens), ints(q_start), 6, 0.01)
    check_attend(got, want, "bf16", 288, 16, U_P["bf16"], FLOOR["bf16"])
    assert np.isneginf(want["lse"][[0, 1, 2, 3, 4, 9, 10, 11, 12]]).all() and np.isfinite(want["lse"][[5, 6, 7, 8]]).all()
    none = uz.latent_attend(q, side.cache, ints(np.zeros((0, 2))), ints([]), ints([0]), 1, 0.01)
    assert (none[0] == 0).all() and torch.isneginf(none[1]).all()
    assert uz.latent_attend(q[:0], side.cache, ints(table), ints(lens), ints(q_start), 6, 0.01)[0].shape == (0, 3, 256)


@pytest.mark.parametrize("fmt", ["e4m3fn", "e5m2"])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("latent,new,heads", [(512, [6, 1], 3), (256, [30, 24], 5), (512, [1, 1], 64), (256, [70, 1], 2)])
def test_attend_nan_and_infinity_reach_only_rows_that_see_them(uz, fmt, kind, latent, new, heads):
    """A latent with a NaN or an infinity makes the rows that see it NaN; what lies past a length, or in a rotary key
    that no row sees, reaches none."""
    g = np.random.default_rng(7)
    at = 200 + new[0] // 2                                                # of the first request: seen by its later rows

    def place(table, i, t):
        return table[i, t // 16], t % 16
    bad = {"e4m3fn": [0x7F], "e5m2": [0x7F, 0x7C, 0xFC]}[fmt]
    for code in bad:
        def edit(side, table, q):
            side.codes[(*place(table, 0, at), 77)] = code
            pg, off = place(table, 1, 150 + new[1] - 1)                   # the last token's page: what lies behind it
            side.codes[pg, off + 1:] = 0x7F
        side, q, table, lens, q_start, scale, want, got = attend_case(uz, 16, latent, 64, heads, kind, fmt, [200, 150], new, edit=edit, seed=8)
        out, lse = got
        sees = np.zeros(sum(new), bool)
        sees[:new[0]] = 200 + np.arange(new[0]) >= at
        assert torch.isnan(out[sees]).all() and torch.isnan(lse[sees]).all()
        keep = {k: v[~sees] for k, v in want.items()}
        check_attend((out[~sees], lse[~sees]), keep, kind, latent + 64, 300, U_P[kind], FLOOR[kind])
        # the first request's rows that do not see it, and all of the second's, as if it were not there
        side.codes[(*place(table, 0, at), 77)] = 0x30
        side.refresh()
        clean = uz.latent_attend(q, side.cache, ints(table), ints(lens), ints(q_start), max(new), scale)
        assert torch.allclose(clean[0][~sees].float(), out[~sees].float(), rtol=2.0 ** -6, atol=float(clean[0].float().abs().max()) * 2.0 ** -6)


def test_attend_nan_rotary_key(uz):
    def edit(side, table, q):
        side.codes[table[0, 3], 5, 256 + 7] = 0x7F                        # token 53
    *_, want, (out, lse) = attend_case(uz, 16, 256, 32, 4, "bf16", "e4m3fn", [50], [8], edit=edit)
    assert torch.isnan(out[3:]).all() and torch.isnan(lse[3:]).all()
    check_attend((out[:3], lse[:3]), {k: v[:3] for k, v in want.items()}, "bf16", 288, 60, U_P["bf16"], FLOOR["bf16"])


@pytest.mark.parametrize("value", ["nan", "inf"])
def test_attend_queries_that_are_not_finite(uz, value):
    def edit(side, table, q):
        q[1, 2, 17] = float(value)
    *_, want, (out, lse) = attend_case(uz, 16, 512, 64, 4, "bf16", "e4m3fn", [50], [3], edit=edit)
    assert torch.isnan(out[1, 2]).all() and not torch.isfinite(lse[1, 2])
    good = np.ones((3, 4), bool)
    good[1, 2] = False
    check_attend((out[torch.from_numpy(good).cuda()][None], lse[torch.from_numpy(good).cuda()][None]), {k: v[good][None] for k, v in want.items()},
                 "bf16", 576, 60, U_P["bf16"], FLOOR["bf16"])


def test_attend_repeats_its_bits_whatever_runs_beside_it(uz):
    side, q, table, lens, q_start, scale, _, got = attend_case(uz, 64, 512, 64, 16, "bf16", "e4m3fn", [3000, 100, 1], [1, 1, 2])
    a = ints(table), ints(lens), ints(q_start)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        both = [uz.latent_attend(q, side.cache, *a, 2, scale, stream=st) for st in streams]
        torch.cuda.synchronize()
        for out, lse in both:
            assert torch.equal(out, got[0]) and torch.equal(lse, got[1])


def test_cache_past_32_bits(uz):
    """Codes past 4 GiB."""
    page, latent, rot, pages = 256, 512, 64, 30000                        # 4.4 GB
    cache = uz.LatentCache.empty(pages, latent, rot, page)
    cache.exps.fill_(120)
    g = np.random.default_rng(9)
    side = Side(uz, 3, page, latent, rot, "e4m3fn", g)
    where = [pages - 1, 29200, 5]
    for i, p in enumerate(where):
        cache.codes[p].copy_(side.cache.codes[i])
        cache.exps[p].copy_(side.cache.exps[i])
    q = rows_of((1, 7, latent + rot), "bf16", g)
    got = uz.latent_attend(q, cache, ints([where]), ints([600]), ints([0, 1]), 1, 0.004)
    want = ref.attend(np_of(q), side.codes, side.exps, latent, "e4m3fn", np.array([[0, 1, 2]]), [600], [0, 1], page, 0.004)
    check_attend(got, want, "bf16", 576, 600, U_P["bf16"], FLOOR["bf16"])
    c, k = rows_of((2, 1, latent), "bf16", g)[:, 0], rows_of((2, 1, rot), "bf16", g)[:, 0]
    uz.latent_store(cache, c, k, ints([0, 0]), dev(freq_of(rot)), torch.tensor([pages * page - 1, 29200 * page + 3], device="cuda"))
    ref.store(side.codes, side.exps, np_of(c), np_of(k), [255, 256 + 3], page, "e4m3fn")
    assert np.array_equal(cache.codes[where].cpu().numpy(), side.codes) and np.array_equal(cache.exps[where].cpu().numpy(), side.exps)
    del cache
    torch.cuda.empty_cache()


# ------------------------------------------------------------------ expanded form
def expanded_case(uz, nope, rot, value, heads, kind, ctx, new, how="", seed=31, pad=0, most=None, scale=None, edit=None):
    g = np.random.default_rng(seed)
    total = [c + n for c, n in zip(ctx, new)]
    rows, keys = sum(new) + pad, sum(max(t, 0) for t in total)
    q, k, v = rows_of((rows, heads, nope + rot), kind, g, how), rows_of((keys, heads, nope), kind, g, how), rows_of((keys, heads, value), kind, g, how)
    r = rows_of((keys, 1, rot), kind, g, how)[:, 0]
    if how == "joined":
        kv = torch.cat([k, v], dim=2)
        k, v = kv[..., :nope], kv[..., nope:]
    q_start, k_start = (np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (new, np.maximum(total, 0)))
    if edit is not None:
        edit(q, k, r, v)
    scale = (nope + rot) ** -0.5 if scale is None else scale
    with np.errstate(invalid="ignore", over="ignore"):
        want = ref.expanded(np_of(q), np_of(k), np_of(r), np_of(v), q_start, k_start, scale)
    out = None
    if how == "odd":
        out = torch.full((rows, heads, value + 3), 7.0, dtype=TYPES[kind], device="cuda")[:, :, 1:value + 1]
    got = uz.latent_attend_expanded(q, k, r, v, ints(q_start), ints(k_start), max(new + [1]) if most is None else most, scale=scale, out=out)
    torch.cuda.synchronize()
    if edit is None:
        check_attend(got, want, kind, nope + rot, max(total + [1]), U_EXPANDED[kind], FLOOR_EXPANDED[kind])
    return q, k, r, v, q_start, k_start, want, got


EXPANDED = [  # nope, rot, value, heads, kind, ctx, new, more
    (128, 64, 128, 1, "bf16", [0], [1], {}),
    (128, 64, 128, 2, "bf16", [0], [130], {}),
    (128, 64, 128, 2, "fp16", [0, 40, 63], [64, 5, 1], dict(how="joined")),
    (64, 32, 64, 3, "bf16", [0, 0, 200], [1, 127, 70], {}),
    (64, 64, 128, 2, "fp16", [10, 300], [129, 33], dict(how="fused")),
    (128, 32, 64, 1, "bf16", [500], [260], dict(how="odd")),
    (64, 32, 128, 5, "fp16", [7, 0, 90], [3, 32, 0], dict(how="odd", pad=2)),
    (128, 64, 64, 1, "bf16", [0, 65], [192, 20], dict(pad=140)),
    (64, 64, 64, 2, "bf16", [1000], [1], {}),
    (128, 64, 128, 2, "bf16", [100], [65], dict(most=1)),
    (64, 32, 64, 2, "fp16", [0], [20], dict(most=5000)),
    (128, 64, 128, 2, "bf16", [30], [40], dict(scale=-2.0)),
    (64, 32, 64, 2, "fp16", [30], [40], dict(scale=4.0)),
]


@pytest.mark.parametrize("case", EXPANDED, ids=str)
def test_expanded(uz, case):
    *args, more = case
    say("expanded", case)
    *_, got = expanded_case(uz, *args, **more)
    if more.get("how") == "odd":
        out = got[0]
        base = torch.as_strided(out, (*out.shape[:2], out.shape[2] + 3), out.stride(), out.storage_offset() - 1)
        assert (base[:, :, 0] == 7).all() and (base[:, :, -2:] == 7).all()


# Heads so many that a workgroup takes 64 rows of one ((rows / 32 + requests + 1) heads above 320), or 128 (of 64 rows: above 560).
MANY_HEADS = [  # nope, rot, value, heads, kind, ctx, new, more
    (128, 64, 128, 60, "bf16", [0], [200], {}),
    (128, 64, 128, 150, "bf16", [0], [200], {}),
    (128, 32, 128, 70, "fp16", [300, 0], [65, 64], dict(how="joined")),
    (128, 64, 64, 130, "fp16", [0, 95, 31], [129, 1, 63], dict(how="fused")),
    (64, 32, 64, 150, "bf16", [700], [130], {}),
    (64, 32, 64, 61, "fp16", [250, 0], [127, 33], dict(how="joined")),
    (64, 64, 128, 140, "bf16", [40], [160], dict(pad=5)),
    (64, 32, 128, 66, "bf16", [128, 127, 129], [33, 34, 1], dict(pad=2)),
    (128, 32, 64, 140, "bf16", [5], [150], dict(scale=-1.0)),
    (128, 64, 128, 64, "bf16", [33], [190], dict(scale=0.0)),
    (64, 64, 64, 150, "fp16", [64], [140], dict(scale=3.0)),
    (64, 64, 64, 64, "bf16", [0], [180], dict(most=64)),
    (128, 64, 128, 140, "fp16", [500, 2], [60, 60], dict(most=60)),
]


@pytest.mark.parametrize("case", MANY_HEADS, ids=str)
def test_expanded_of_many_heads(uz, case):
    *args, more = case
    say("expanded", case)
    expanded_case(uz, *args, **more)


@pytest.mark.parametrize("heads", [64, 150])
@pytest.mark.parametrize("nope,rot,value,kind", [(128, 64, 128, "bf16"), (64, 32, 64, "fp16"), (64, 64, 128, "bf16")])
def test_expanded_of_many_heads_with_values_that_are_not_finite(uz, nope, rot, value, kind, heads):
    """As if the tokens were not there, but for the rows and channels that see them."""
    inf = float("inf")

    def edit(q, k, r, v):
        v[70, 3, 5], v[100, 3, 6], v[149, 9, 40] = float("nan"), inf, -inf
        k[120, 7, 11] = float("nan")
    *_, want, (out, lse) = expanded_case(uz, nope, rot, value, heads, kind, [10], [140], edit=edit)
    at = 10 + np.arange(140)
    odd = np.zeros(out.shape, bool)
    odd[at >= 70, 3, 5] = odd[at >= 100, 3, 6] = odd[at >= 149, 9, 40] = odd[at >= 120, 7] = True
    assert torch.isnan(out[torch.from_numpy(at >= 70), 3, 5]).all() and (out[torch.from_numpy(at >= 100), 3, 6] == inf).all()
    assert (out[torch.from_numpy(at >= 149), 9, 40] == -inf).all() and torch.isnan(out[torch.from_numpy(at >= 120), 7]).all()
    assert torch.isnan(lse[torch.from_numpy(at >= 120), 7]).all()
    gone = torch.from_numpy(odd).cuda()
    plain = {k: v.copy() if isinstance(v, np.ndarray) else v for k, v in want.items()}
    for name in ("out", "spread", "floor"):
        plain[name] = np.where(odd, 0.0, np.broadcast_to(plain[name], odd.shape) if np.ndim(plain[name]) else plain[name])
    whole = odd.all(axis=2)
    plain["lse"] = np.where(whole, 0.0, plain["lse"])
    plain["size"] = np.where(whole, 0.0, np.broadcast_to(plain["size"], whole.shape))
    check_attend((torch.where(gone, torch.zeros_like(out), out), torch.where(torch.from_numpy(whole).cuda(), torch.zeros_like(lse), lse)), plain, kind,
                 nope + rot, 150, U_EXPANDED[kind], FLOOR_EXPANDED[kind])


@pytest.mark.parametrize("heads", [2, 64, 150])
def test_expanded_values_near_the_largest(uz, heads):
    """Sums of values that 32 bits hold one by one, but not added up: divided first, they are within the type."""
    def edit(q, k, r, v):
        v.mul_(2.0 ** 126 / v.abs().max())
    *_, want, (out, lse) = expanded_case(uz, 128, 64, 128, heads, "bf16", [60], [140], edit=edit)
    check_attend((out, lse), want, "bf16", 192, 200, U_EXPANDED["bf16"], FLOOR_EXPANDED["bf16"])


def test_expanded_many_requests(uz):
    expanded_case(uz, 64, 32, 64, 1, "bf16", [0] * 150, [1, 2, 0] * 50)


def test_expanded_rows_without_keys(uz):
    """More rows than keys: the first see nothing; no keys, no requests, no rows."""
    g = np.random.default_rng(32)
    q, k, v, r = rows_of((9, 2, 96), "bf16", g), rows_of((4, 2, 64), "bf16", g), rows_of((4, 2, 64), "bf16", g), rows_of((4, 1, 32), "bf16", g)[:, 0]
    want = ref.expanded(np_of(q), np_of(k), np_of(r), np_of(v), [0, 6, 8], [0, 4, 4], 0.1)
    got = uz.latent_attend_expanded(q, k, r, v, ints([0, 6, 8]), ints([0, 4, 4]), 6, scale=0.1)
    check_attend(got, want, "bf16", 96, 4, U_EXPANDED["bf16"], 0.0)
    assert np.isneginf(want["lse"][[0, 1, 6, 7, 8]]).all() and np.isfinite(want["lse"][2:6]).all()
    none = uz.latent_attend_expanded(q, k[:0], r[:0], v[:0], ints([0, 9]), ints([0, 0]), 9)
    assert (none[0] == 0).all() and torch.isneginf(none[1]).all()
    none = uz.latent_attend_expanded(q, k, r, v, ints([0]), ints([0]), 9)
    assert (none[0] == 0).all() and torch.isneginf(none[1]).all()
    assert uz.latent_attend_expanded(q[:0], k, r, v, ints([0, 0]), ints([0, 4]), 9)[0].shape == (0, 2, 64)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("value", [64, 128])
def test_expanded_nan_and_infinity_reach_only_rows_that_see_them(uz, kind, value):
    """In values: their channel of the rows that see them; in keys: those rows whole."""
    inf = float("inf")

    def edit(q, k, r, v):
        v[50, 0, 3], v[70, 0, 3] = inf, -inf
        v[90, 0, 10] = float("nan")
        v[100, 0, 20] = -inf
        v[260, 1, 5] = inf                                                # the second request's
        k[120, 1, 7] = float("nan")
    *_, want, (out, lse) = expanded_case(uz, 64, 32, value, 2, kind, [40, 5], [160, 80], edit=edit)
    place = np.concatenate([np.arange(40, 200), np.arange(205, 285)])     # in the joined keys
    first = np.arange(240) < 160
    o = out.float().cpu().numpy()
    for ch, at, what in [(3, 50, inf), (20, 100, -inf)]:
        rows = first & (place >= at) & ((ch != 3) | (place < 70))
        assert (o[rows, 0, ch] == what).all() and np.isfinite(o[first & (place < at), 0, ch]).all()
    assert np.isnan(o[first & (place >= 70), 0, 3]).all() and np.isnan(o[first & (place >= 90), 0, 10]).all()
    assert np.isfinite(o[first & (place < 90), 0, 10]).all()
    rows = ~first & (place >= 260)
    assert (o[rows, 1, 5] == inf).all()
    assert np.isnan(o[first & (place >= 120), 1]).all() and np.isnan(lse[:160][place[:160] >= 120, 1].cpu().numpy()).all()
    good = np.isfinite(want["out"]) & np.isfinite(o)
    # every other number is as it should be
    hit = np.zeros_like(good)
    hit[first, 0, 3], hit[first, 0, 10], hit[first, 0, 20], hit[~first, 1, 5] = (place >= 50)[first], (place >= 90)[first], (place >= 100)[first], rows[~first]
    hit[first & (place >= 120), 1] = True
    assert (np.isfinite(o) == ~hit).all()
    with np.errstate(invalid="ignore"):
        tol = U_OUT[kind] * np.abs(want["out"]) + (U_EXPANDED[kind] + 2.0 ** -10) * want["spread"] + FLOOR_EXPANDED[kind] * want["floor"]
        assert (np.abs(o - want["out"])[~hit] <= tol[~hit]).all()


def test_expanded_repeats_its_bits_on_another_stream_and_in_a_graph(uz):
    q, k, r, v, q_start, k_start, _, got = expanded_case(uz, 128, 64, 128, 2, "bf16", [70, 0], [200, 33])
    a = ints(q_start), ints(k_start)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    there = uz.latent_attend_expanded(q, k, r, v, *a, 200, stream=side)
    side.synchronize()
    assert torch.equal(there[0], got[0]) and torch.equal(there[1], got[1])
    out, lse = torch.zeros_like(got[0]), torch.zeros_like(got[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        uz.latent_attend_expanded(q, k, r, v, *a, 200, out=out, lse=lse)
    for turn in range(3):
        q.normal_()
        a[0].copy_(ints([0, 200 - turn, 233]))
        graph.replay()
        torch.cuda.synchronize()
        want = uz.latent_attend_expanded(q, k, r, v, *a, 200)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]), turn


# ------------------------------------------------------------------ together
def test_both_forms_agree_and_steps_run_in_a_graph(uz):
    """A prompt in the expanded form, its latents stored, then single tokens in the absorbed form, in a graph: as the
    expanded form over the same, rounded latents."""
    g = np.random.default_rng(41)
    heads, nope, rot, value, latent, page, reqs = 4, 64, 32, 64, 256, 16, 3
    freq, scale = dev(freq_of(rot)), (nope + rot) ** -0.5
    up_k, up_v = (torch.from_numpy(g.standard_normal((heads, latent, n)).astype(np.float32)).cuda() * latent ** -0.5 for n in (nope, value))
    cache = uz.LatentCache.empty(60, latent, rot, page)
    table = ints(np.full((reqs, 20), -1))
    prompts = [40, 1, 130]
    old, new, free = ints([0] * reqs), ints(prompts), ints(g.permutation(60))
    rows = sum(prompts)

    def token(rows):
        return (rows_of((rows, 1, latent), "bf16", g)[:, 0], rows_of((rows, 1, rot), "bf16", g)[:, 0], rows_of((rows, heads, nope + rot), "bf16", g))
    c, k_rot, q = token(rows)
    plan = uz.kv_plan(old, new, free, table, page, rows)
    places = uz.kv_positions(plan.lens, plan.q_start, rows)
    q = uz.rotate(q, places, freq, first=nope)
    uz.latent_store(cache, c, k_rot, places, freq, plan.slots)
    turned = uz.rotate(k_rot[:, None], places, freq)[:, 0]
    k, v = (torch.matmul(c.float(), w).transpose(0, 1).to(torch.bfloat16) for w in (up_k, up_v))
    out, _ = uz.latent_attend_expanded(q, k, turned, v, plan.q_start, plan.q_start, max(prompts))

    def absorbed(q):
        return torch.cat([torch.matmul(q[..., :nope].float().transpose(0, 1), up_k.transpose(1, 2).contiguous()).transpose(0, 1).to(torch.bfloat16),
                          q[..., nope:]], dim=-1)
    lat, _ = uz.latent_attend(absorbed(q), cache, table, plan.lens, plan.q_start, max(prompts), scale)
    from_latents = torch.matmul(lat.float().transpose(0, 1), up_v).transpose(0, 1)
    # the two differ by the latents' rounding to 8 bits, 2^-4 of each value, and some of the queries' and keys'
    assert (out.float() - from_latents).norm() < 2.0 ** -4 * 1.5 * out.float().norm()

    used = int(plan.counts[0])
    step_plan = uz.kv_plan_buffers(reqs, reqs, page)
    one, fr = ints([1] * reqs), free[used:used + reqs].clone()
    at = plan.lens.clone()
    c, k_rot, q = token(reqs)
    q_abs = absorbed(q)
    place = ints([0] * reqs)
    res, lse = torch.zeros(reqs, heads, latent, dtype=torch.bfloat16, device="cuda"), torch.zeros(reqs, heads, device="cuda")
    ws = uz.latent_attend_workspace(q_abs, cache, reqs, 1)

    def step():
        uz.kv_plan(at, one, fr, table, page, reqs, out=step_plan)
        uz.kv_positions(step_plan.lens, step_plan.q_start, reqs, out=place)
        uz.latent_store(cache, c, k_rot, place, freq, step_plan.slots, q=q[..., nope:], q_out=q_abs[..., latent:])
        uz.latent_attend(q_abs, cache, table, step_plan.lens, step_plan.q_start, 1, scale, out=res, lse=lse, ws=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(20):
        for t, x in zip((c, k_rot, q), token(reqs)):
            t.copy_(x)
        q_abs.copy_(absorbed(q))
        fr.copy_(free[used:used + reqs])
        graph.replay()
        torch.cuda.synchronize()
        lens = step_plan.lens.cpu().numpy()
        assert np.array_equal(lens, np.array(prompts) + turn + 1) and place.tolist() == [n - 1 for n in lens]
        codes, exps = cache.codes.cpu().numpy(), cache.exps.cpu().numpy()
        want = ref.attend(np_of(q_abs), codes, exps, latent, "e4m3fn", table.cpu().numpy(), lens, [0, 1, 2, 3], page, scale)
        check_attend((res, lse), want, "bf16", latent + rot, int(lens.max()), U_P["bf16"], FLOOR["bf16"])
        used += int(step_plan.counts[0])
        at.copy_(step_plan.lens)


def test_workspaces_of_two_graphs(uz):
    """Two captured calls that share a workspace, replayed one after the other."""
    side, q, table, lens, q_start, scale, _, got = attend_case(uz, 64, 256, 64, 16, "bf16", "e4m3fn", [2000, 100], [1, 1])
    other = rows_of(tuple(q.shape), "bf16", np.random.default_rng(3))
    a = ints(table), ints(lens), ints(q_start)
    ws = uz.latent_attend_workspace(q, side.cache, 2, 1)
    want = uz.latent_attend(other, side.cache, *a, 1, scale)
    graphs = []
    for x in (q, other):
        o, s = torch.zeros_like(got[0]), torch.zeros_like(got[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            uz.latent_attend(x, side.cache, *a, 1, scale, out=o, lse=s, ws=ws)
        graphs.append((graph, o, s))
    for _ in range(3):
        for (graph, o, s), w in zip(graphs, (got, want)):
            o.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, w[0]) and torch.equal(s, w[1])


def test_refusals(uz):
    c = uz.LatentCache.empty(2, 256, 32, 16)
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")  # noqa: E731
    for args in [(u8(2, 16, 288).cpu(), u8(2, 16, 2), 32), (u8(2, 16, 288), u8(2, 16), 32), (u8(2, 16, 288), u8(2, 16, 2), 288),
                 (u8(2, 16, 288), u8(2, 16, 2), 0), (u8(2, 16, 576)[..., ::2], u8(2, 16, 2), 32), (u8(2, 16, 288), u8(2, 16, 2), 32, "bf16")]:
        with pytest.raises(ValueError):
            uz.LatentCache(*args)
    q = torch.zeros(2, 3, 288, dtype=torch.bfloat16, device="cuda")
    t, n, s = ints([[0]]), ints([2]), ints([0, 2])
    lse = torch.zeros(2, 3, device="cuda")
    for b in [dict(q=q.float()), dict(q=q.double()), dict(q=q[..., :256]), dict(q=q.cpu()), dict(lens=n.long()), dict(q_start=s[:1]), dict(table=t[0]),
              dict(out=q), dict(out=q[..., :256].half()), dict(lse=lse.half()), dict(lse=lse[:1]), dict(max_new=-1)]:
        a = {"q": q, "table": t, "lens": n, "q_start": s, "max_new": 2, "out": None, "lse": None, **b}
        with pytest.raises(ValueError):
            uz.latent_attend(a["q"], c, a["table"], a["lens"], a["q_start"], a["max_new"], 0.1, out=a["out"], lse=a["lse"])
    with pytest.raises(ValueError):
        uz.latent_attend(q.clone().requires_grad_(True), c, t, n, s, 2, 0.1)
    with pytest.raises(uz.UzipError) as e:
        uz.latent_attend(q, c, t, n, s, 2, 0.1, ws=u8(16))
    assert e.value.status == uz.ENOSPC
    for scale in (float("nan"), float("inf")):
        with pytest.raises(uz.UzipError):
            uz.latent_attend(q, c, t, n, s, 2, scale)
    odd = uz.LatentCache.empty(2, 128, 32, 16)                            # a width that has no kernel
    with pytest.raises(uz.UzipError):
        uz.latent_attend(q[..., :160], odd, t, n, s, 2, 0.1, ws=u8(1 << 20))
    x, r, f, p = torch.zeros(2, 256, device="cuda"), torch.zeros(2, 32, device="cuda"), dev(freq_of(32)), ints([0, 0])
    slots = torch.zeros(2, dtype=torch.int64, device="cuda")
    for b in [dict(x=x[:1]), dict(x=x.half()), dict(x=x[:, :128]), dict(r=r[..., ::2]), dict(f=dev(freq_of(64))), dict(p=p[:1]), dict(slots=slots[:1]),
              dict(slots=slots.int()), dict(q=torch.zeros(2, 1, 64, device="cuda")), dict(q_out=torch.zeros(2, 1, 32, device="cuda")),
              dict(x=x.clone().requires_grad_(True))]:
        a = {"x": x, "r": r, "f": f, "p": p, "slots": slots, "q": None, "q_out": None, **b}
        with pytest.raises(ValueError):
            uz.latent_store(c, a["x"], a["r"], a["p"], a["f"], a["slots"], q=a["q"], q_out=a["q_out"])
    h = lambda *s: torch.zeros(*s, dtype=torch.float16, device="cuda")  # noqa: E731
    good = {"q": h(4, 2, 96), "k": h(4, 2, 64), "r": h(4, 32), "v": h(4, 2, 64), "qs": ints([0, 4]), "ks": ints([0, 4]), "out": None, "lse": None}
    for b in [dict(q=h(4, 2, 64)), dict(k=h(3, 2, 64)), dict(k=h(4, 1, 64)), dict(v=h(4, 2, 64).float()), dict(r=h(4, 1, 32)), dict(qs=ints([0])),
              dict(ks=ints([])), dict(out=h(4, 2, 32)), dict(lse=h(4, 2)), dict(v=h(4, 64, 2).transpose(1, 2)), dict(k=h(4, 2, 64).requires_grad_(True))]:
        a = {**good, **b}
        with pytest.raises(ValueError):
            uz.latent_attend_expanded(a["q"], a["k"], a["r"], a["v"], a["qs"], a["ks"], 4, out=a["out"], lse=a["lse"])
    with pytest.raises(uz.UzipError):
        uz.latent_attend_expanded(h(4, 2, 80), h(4, 2, 48), h(4, 32), h(4, 2, 64), ints([0, 4]), ints([0, 4]), 4)
