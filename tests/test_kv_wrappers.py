"""The key/value cache's Python wrappers without a GPU: sizes that do not fit the C call's 32 bits are refused, not
taken for what is left of them."""
import pytest


@pytest.fixture(scope="module")
def uz():
    import paper_2604_17172_amd as m
    return m


@pytest.mark.parametrize("requests,rows,page", [(1, (1 << 32) + 5, 16), ((1 << 32) + 1, 5, 16), (1, 5, (1 << 32) + 16), (1, 1 << 22 | 1, 16),
                                                (4097, 5, 16), (-1, 5, 16), (1, -(1 << 32) + 5, 16), (1, 5, -(1 << 32) + 16), (1, 5, 24)])
def test_plan_sizes_out_of_range(uz, requests, rows, page):
    with pytest.raises(uz.UzipError) as e:
        uz.kv_plan_buffers(requests, rows, page, device="meta")
    assert e.value.status == uz.EINVAL


def test_plan_sizes_at_their_ends(uz):
    for requests, rows, page in [(0, 0, 16), (uz.KV_MAX_REQUESTS, uz.KV_MAX_ROWS, 16), (1, 1, 256)]:
        plan = uz.kv_plan_buffers(requests, rows, page, device="meta")
        assert plan.slots.shape == (rows,) and plan.q_start.shape == (requests + 1,)
        assert plan.runs.shape == (uz.uzip_kv_max_runs(rows, requests, page), 2)
