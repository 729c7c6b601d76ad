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
