"""pd_attn_chunk where it can go wrong: units of a single tile, groups that do not divide evenly, scales of V at the ends of their range.

Bounds are those of test_gpu_chunk."""
import numpy as np
import pytest
import torch

from test_gpu_chunk import check, queries
from test_gpu_rope import Pages, i32, offsets

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2512_19720_b200 import api
    return api


@pytest.mark.parametrize("hq,hkv,d", [(64, 2, 64), (17, 1, 128)])
@pytest.mark.parametrize("between", [[], [130], [3], [9, 40]], ids=str)
def test_units_of_one_tile_behind_each_other(api, between, hq, hkv, d):
    """Units of a single tile, all of it one slot's, behind units of their own kind and of the others: no slot loses count of the units."""
    new = ([1] * 5 + between) * 60
    lens = [n + h for n, h in zip(new, np.random.default_rng(3).integers(0, 100, len(new)).tolist())]
    pages = Pages(lens, hkv, d, 64, 11)
    q = queries(sum(new), hq, d, torch.float16, 7)
    first = check(api, pages, q, lens, new, only=set(range(0, sum(new), 7)))
    for _ in range(30):
        assert torch.equal(first, api.pd_attn_chunk(q, *pages.tensors(), offsets(new), i32(lens), pages.block_table))
    assert api.pd_device_status(api.chunk_workspace()) == 0


@pytest.mark.parametrize("hq,hkv", [(129, 1), (258, 2), (257, 1), (514, 2)])
@pytest.mark.parametrize("new,held", [([3], [200]), ([5, 1], [60, 1000])], ids=str)
def test_groups_that_do_not_divide_evenly(api, new, held, hq, hkv):
    """More than 128 query heads share a key/value head and their last share is smaller: rows that stand for no head hold the next
    key/value head's queries, or nothing, and have no say."""
    lens = [a + b for a, b in zip(held, new)]
    for dtype in TYPES:
        pages = Pages(lens, hkv, 64, 16, 13)
        q = queries(sum(new), hq, 64, dtype, 17)
        first = check(api, pages, q, lens, new)
        if hkv == 1:
            continue
        for other in (float("inf"), -300.0, 300.0):
            changed = q.clone()
            changed[:, hq // 2:] *= other
            got = api.pd_attn_chunk(changed, *pages.tensors(), offsets(new), i32(lens), pages.block_table)
            assert torch.equal(got[:, :hq // 2], first[:, :hq // 2])
