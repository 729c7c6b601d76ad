"""GPU: the 8-bit key/value cache at its edges."""
import numpy as np
import pytest
import torch

from oracle import kv as ref
from test_gpu_kv import Side, TYPES, check_attend, dev, ints, np_of, rows_of, run_attend, say, uz  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ plan
def test_a_plan_used_again_has_the_status_of_its_last_call(uz):
    plan = uz.kv_plan_buffers(2, 64, 16)
    old, table = ints([0, 0]), ints(np.full((2, 3), -1))
    few, enough = ints([5]), ints([5, 6, 7])
    for _ in range(2):
        uz.kv_plan(old, ints([16, 17]), few, table, 16, 33, out=plan)     # the second request finds no pages
        torch.cuda.synchronize()
        assert int(plan.status.item()) == uz.ENOSPC and plan.lens.tolist() == [16, 0]
        with pytest.raises(uz.UzipError) as e:
            uz.kv_plan(old, ints([16, 17]), few, table, 16, 33, out=plan, check=True)
        assert e.value.status == uz.ENOSPC
        uz.kv_plan(old, ints([16, 17]), enough, table, 16, 33, out=plan, check=True)
        assert int(plan.status.item()) == uz.OK and plan.lens.tolist() == [16, 17]
        with pytest.raises(uz.UzipError) as e:
            uz.kv_plan(old, ints([16, -1]), enough, table, 16, 33, out=plan, check=True)
        assert e.value.status == uz.EINVAL
    uz.kv_plan(old, ints([0, 0]), enough, table, 16, 0, out=plan, check=True)
    plan.status.fill_(77)                                                 # whatever it held
    uz.kv_plan(old, ints([16, 0]), enough, table, 16, 64, out=plan, check=True)
    uz.kv_plan(ints([]), ints([]), enough, table[:0], 16, 5, out=plan, check=True)


def test_each_replay_of_a_plan_has_its_own_status(uz):
    plan = uz.kv_plan_buffers(1, 600, 16)
    old, new, free, table = ints([0]), ints([16]), ints([3]), ints([[-1, -1]])
    uz.kv_plan(old, new, free, table, 16, 600, out=plan)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        uz.kv_plan(old, new, free, table, 16, 600, out=plan)              # three workgroups
    for tokens, status in ((16, uz.OK), (32, uz.ENOSPC), (16, uz.OK), (-1, uz.EINVAL), (48, uz.ENOSPC), (1, uz.OK)):
        new.fill_(tokens)
        graph.replay()
        torch.cuda.synchronize()
        assert int(plan.status.item()) == status, tokens


def test_a_plan_used_again_for_fewer_requests_shows_only_theirs(uz):
    """Eight requests take three tokens each, then five of them one: attention over the plan's lengths sees no request of before."""
    g = np.random.default_rng(94)
    side = Side(uz, 16, 1, 16, 64, "e4m3fn", g)
    plan = uz.kv_plan_buffers(8, 24, 16)
    free, table = ints(np.arange(16)), ints(np.full((8, 2), -1))
    uz.kv_plan(ints([0] * 8), ints([3] * 8), free, table, 16, 24, out=plan, check=True)
    k, kd = rows_of((24, 1, 64), "bf16", g)
    v, vd = rows_of((24, 1, 64), "bf16", g)
    uz.kv_store(side.cache, kd, vd, plan.slots, plan.runs, plan.counts)
    side.store(np_of(k), np_of(v), plan.slots.tolist(), [(3 * i, 3) for i in range(8)])
    uz.kv_plan(ints([3] * 5), ints([1] * 5), free, table[:5], 16, 5, out=plan, check=True)
    assert plan.lens.tolist() == [4] * 5 and plan.q_start.tolist() == list(range(6)) and plan.slots.shape == (5,)
    k, kd = rows_of((5, 1, 64), "bf16", g)
    v, vd = rows_of((5, 1, 64), "bf16", g)
    uz.kv_store(side.cache, kd, vd, plan.slots, plan.runs, plan.counts)
    side.store(np_of(k), np_of(v), plan.slots.tolist(), [(i, 1) for i in range(5)])
    q, qd = rows_of((5, 2, 64), "bf16", g)
    want = ref.attend(np_of(q), side.k, side.k_exp, side.v, side.v_exp, "e4m3fn", table.cpu().numpy(), [4] * 5, range(6), 16, 0.3)
    got = uz.kv_attend(qd, side.cache, table, plan.lens, plan.q_start, 1, scale=0.3)
    check_attend(got, want, "bf16", 64, 4)
    uz.kv_plan(ints([4] * 8), ints([2] * 8), free, table, 16, 24, out=plan, check=True)
    assert plan.lens.tolist() == [6] * 8 and plan.q_start.tolist() == list(range(0, 18, 2)) and plan.slots.shape == (24,)


# ------------------------------------------------------------------ attention: chosen scores and values
class Scored(Side):
    """One request of `total` tokens, one head: token t scores scores[t] (else 0) for a query that is 1 in channel 0."""

    def __init__(self, uz, fmt, total, dim, scores, page=16, seed=91):
        g = np.random.default_rng(seed)
        pages = -(-total // page)
        super().__init__(uz, pages, 1, page, dim, fmt, g)
        self.total, self.table = total, g.permutation(pages).astype(np.int32)[None]
        self.k[:], self.k_exp[:], self.v_exp[:] = 0, 127, 127
        self.v[:] = ref.encode(g.standard_normal(self.v.shape), fmt)
        for t, s in scores.items():
            self.k[self.at(t)][0] = ref.encode(s, fmt)
        self.g = g

    def at(self, t):
        return self.table[0, t // self.page], 0, t % self.page

    def value(self, t, ch, x):
        self.v[self.at(t)][ch] = ref.encode(x, self.fmt)

    def attend(self, uz, kind, new, window=0, group=1):
        for mine, its in ((self.k, self.cache.k), (self.v.transpose(0, 1, 3, 2), self.cache.v), (self.k_exp, self.cache.k_exp),
                          (self.v_exp, self.cache.v_exp)):
            its.copy_(dev(mine))
        q, qd = rows_of((new, group, self.dim), kind, self.g)
        q[:, :, 0] = 1
        qd[:, :, 0] = 1
        with np.errstate(invalid="ignore"):
            want = ref.attend(np_of(q), self.k, self.k_exp, self.v, self.v_exp, self.fmt, self.table, [self.total], [0, new],
                              self.page, 1.0, window)
        return want, run_attend(uz, self, qd, ints(self.table), ints([self.total]), ints([0, new]), new, 1.0, window)


@pytest.mark.parametrize("fmt", ["e4m3fn", "e5m2"])
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("total,new", [(300, 1), (321, 1), (330, 10), (530, 200), (5000, 2)])
def test_attend_values_near_the_end_of_32_bits(uz, fmt, kind, total, new):
    """A token that scores 5 (a factor of 2^7.2) more than those before it, with values of 2^127: sums whose single weights are
    at most 1 stay finite, whichever step the token comes in."""
    say("large values", fmt, kind, total, new)
    top, last = ref.FORMATS[fmt][2], ref.FORMATS[fmt][3]
    for hot, score in ((5, 0.0), (70, 5.0), (261, 5.0), (total - new, 5.0)):
        side = Scored(uz, fmt, total, 64, {hot: score})
        pg = side.at(hot)[0]
        side.v[pg] = 0
        side.v_exp[pg] = last
        for ch in range(0, 64, 3):
            side.value(hot, ch, -top if ch % 2 else top)
        want, got = side.attend(uz, kind, new)
        assert np.isfinite(want["out"]).all() and np.abs(want["out"]).max() > 1e34
        check_attend(got, want, kind, 64, total)


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("total,new,window", [(300, 1, 0), (321, 9, 0), (530, 200, 0), (530, 200, 450), (3000, 1, 0), (9000, 170, 0)])
def test_attend_infinity_at_a_weight_below_32_bits(uz, kind, total, new, window):
    """An infinite value is infinite for every row that sees it, also where its weight of e^-256 is 0 in 32 bits, and
    whichever step, wave or piece it falls in."""
    say("infinity", kind, total, new, window)
    for most in (90, 130, 259, total - new - 3):                          # the token that has all the weight
        side = Scored(uz, "e5m2", total, 64, {most: 256.0})
        for t, ch, x in [(5, 3, "inf"), (89, 4, "-inf"), (91, 8, "inf"), (200, 5, "inf"), (201, 5, "-inf"), (270, 9, "-inf"),
                         (total - 1, 6, "inf"), (100, 7, "nan"), (total - new, 10, "inf"), (total // 2, 11, "-inf")]:
            side.value(t, ch, float(x))
        want, (out, lse) = side.attend(uz, kind, new, window)
        got, fine = np_of(out), np.isfinite(want["out"])
        assert not fine.all() and fine.any()
        assert np.array_equal(got[~fine], want["out"][~fine], equal_nan=True)
        assert np.isfinite(got[fine]).all()
        clean = {k: np.where(fine, v, 0.0) if k in ("out", "spread") else v for k, v in want.items()}
        check_attend((torch.from_numpy(np.where(fine, got, 0.0)), lse), clean, kind, 64, total)


# ------------------------------------------------------------------ attention: memory beside the outputs
def between_guards(shape, dtype, fill=77):
    """A contiguous tensor with 4096 guard bytes before and behind it, and a check of them."""
    size = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
    room = torch.full((size + 8192,), fill, dtype=torch.uint8, device="cuda")

    def check():
        assert (room[:4096] == fill).all() and (room[4096 + size:] == fill).all()
    return room[4096:4096 + size].view(dtype).view(shape), check


@pytest.mark.parametrize("starts", [[0, 300, 0, 300, 0, 300], [300, 200, 100, 50, 20, 0], [-5, 2 ** 31 - 1, -2 ** 31, 7, 7, 301],
                                    [0, 0, 0, 0, 0, 0], [299, 299, 300, 2 ** 30, 0, 1]], ids=str)
@pytest.mark.parametrize("kind,dim,heads", [("bf16", 128, 8), ("fp16", 64, 2), ("fp32", 96, 4)])
def test_attend_writes_only_its_outputs_whatever_the_row_starts(uz, kind, dim, heads, starts):
    """Row starts that descend, repeat, share rows or lie outside: nothing beside out, lse and workspace is written."""
    say("row starts", starts, kind, dim)
    g = np.random.default_rng(95)
    side = Side(uz, 40, 1, 64, dim, "e4m3fn", g)
    q, qd = rows_of((300, heads, dim), kind, g)
    for lens in ([2500, 2500, 700, 2 ** 31 - 1, -4], [300] * 5):
        out, out_fine = between_guards((300, heads, dim), TYPES[kind])
        lse, lse_fine = between_guards((300, heads), torch.float32)
        for most in (1, 60, 300):
            ws, ws_fine = between_guards((uz.uzip_kv_attend_workspace({"bf16": 0, "fp16": 1, "fp32": 2}[kind], 300, heads, 1, dim, 5, most),),
                                         torch.uint8)
            table = torch.randint(-1, 40, (5, 40), dtype=torch.int32, device="cuda")
            uz.kv_attend(qd, side.cache, table, ints(lens), ints(starts), most, out=out, lse=lse, ws=ws)
            torch.cuda.synchronize()
            out_fine()
            lse_fine()
            ws_fine()


# ------------------------------------------------------------------ attention: pieces longer than the least
def check_sampled(uz, kind, dim, kv, group, fmt, page, ctx, new, seed, window=0):
    """All requests read pages of one small pool; out, lse and a workspace of just its size lie between guards; a few rows of
    each of a few requests are compared."""
    g = np.random.default_rng(seed)
    most = max(c + n for c, n in zip(ctx, new))
    pages = -(-most // page) + 7
    side = Side(uz, pages, kv, page, dim, fmt, g)
    finite = np.arange(256, dtype=np.uint8)[np.isfinite(ref.code_values(fmt)) & (np.abs(ref.code_values(fmt)) < 8)]
    side.k, side.v = finite[side.k % len(finite)], finite[side.v % len(finite)]
    side.k_exp[:], side.v_exp[:] = g.integers(124, 129, side.k_exp.shape), g.integers(124, 129, side.v_exp.shape)
    for mine, its in ((side.k, side.cache.k), (side.v.transpose(0, 1, 3, 2), side.cache.v), (side.k_exp, side.cache.k_exp),
                      (side.v_exp, side.cache.v_exp)):
        its.copy_(dev(mine))
    table = np.stack([g.permutation(pages)[:pages - 6] for _ in ctx]).astype(np.int32)
    lens = np.array([c + n for c, n in zip(ctx, new)], np.int32)
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    rows, heads = sum(new), kv * group
    q, qd = rows_of((rows, heads, dim), kind, g)
    out, out_fine = between_guards((rows, heads, dim), TYPES[kind])
    lse, lse_fine = between_guards((rows, heads), torch.float32)
    ws, ws_fine = between_guards((uz.kv_attend_workspace(qd, side.cache, len(ctx), max(new)).numel(),), torch.uint8, fill=255)
    ws.fill_(255)
    scale = dim ** -0.5
    uz.kv_attend(qd, side.cache, ints(table), ints(lens), ints(starts), max(new), scale=scale, window=window, out=out, lse=lse, ws=ws)
    torch.cuda.synchronize()
    out_fine()
    lse_fine()
    ws_fine()
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    for i in sorted({0, len(ctx) - 1, *g.integers(0, len(ctx), 3).tolist()}):
        for j in sorted({0, new[i] - 1, *g.integers(0, new[i], 3).tolist()}):
            r, length = int(starts[i]) + j, ctx[i] + j + 1                # the row as the last of a shorter request
            want = ref.attend(np_of(q[r:r + 1]), side.k, side.k_exp, side.v, side.v_exp, fmt, table[i:i + 1], [length], [0, 1], page,
                              scale, window)
            check_attend((out[r:r + 1], lse[r:r + 1]), want, kind, dim, length)


@pytest.mark.parametrize("kind,dim,kv,group,ctx,new", [
    ("bf16", 128, 8, 1, [14000], [520]),                                  # 40 blocks of 228 steps: pieces of 18
    ("fp16", 64, 8, 2, [14000, 9000], [300, 201]),                        # 72 blocks: pieces of 13 or 14
    ("bf16", 96, 4, 3, [60000, 100, 3], [200, 1, 180]),                   # long and short lists in one call
    ("fp16", 256, 2, 4, [20000, 20], [240, 40]),
    ("bf16", 192, 2, 4, [20000, 777], [400, 3]),
])
def test_attend_long_pieces_of_many_rows(uz, kind, dim, kv, group, ctx, new):
    say("long pieces", kind, dim, kv, group, ctx, new)
    check_sampled(uz, kind, dim, kv, group, "e4m3fn", 64, ctx, new, 96)
    check_sampled(uz, kind, dim, kv, group, "e5m2", 16, ctx, new, 97, window=9000)


@pytest.mark.parametrize("kind,dim,group", [("bf16", 128, 4), ("fp16", 64, 7), ("fp32", 96, 1), ("bf16", 64, 20), ("fp32", 256, 2)])
def test_attend_long_pieces_of_few_rows(uz, kind, dim, group):
    """More than 32768 steps in all: four pieces for a compute unit are longer than 32 steps."""
    say("long few", kind, dim, group)
    ctx = [5000 + 101 * i for i in range(64)]
    check_sampled(uz, kind, dim, 8, group, "e4m3fn", 64, ctx, [1] * 64, 98)
    check_sampled(uz, kind, dim, 8, group, "e5m2", 128, ctx, [1] * 40 + [2] * 24, 99, window=7777)
