"""GPU: the 8-bit key/value cache at its edges."""
import numpy as np
import pytest
import torch

from test_gpu_kv import ints, uz  # noqa: F401

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
