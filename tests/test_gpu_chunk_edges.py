"""pd_attn_chunk where it can go wrong: units of a single tile, groups that do not divide evenly, scales of V at the ends of their range.

Bounds are those of test_gpu_chunk."""
import numpy as np
import pytest
import torch

from test_gpu_chunk import UNIT, check, definition, f64, queries
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


# ------------------------------------------------------------------ scales of V at the ends of their range
def check_what_is_attended_to(api, pages, q, lens, new, max_new=0, scale=None, rows=None):
    """test_gpu_chunk's bound with nothing in it of keys that a token does not attend to: each of the tokens `rows` as the last one of a sequence.
    Room for u of the bound beside it: it is E + u |want| with all errors E before the output is rounded, but what is rounded is the sum, up to
    |want| + E, which counts where large terms cancel that weights in binary16 have lost."""
    scale = q.shape[2] ** -0.5 if scale is None else scale
    got = api.pd_attn_chunk(q, *pages.tensors(), offsets(new), i32(lens), pages.block_table, max_new, scale)
    assert api.pd_device_status(api.chunk_workspace()) == 0
    at = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        one = Pages.__new__(Pages)
        one.page, one.codes, one.scales, one.table = pages.page, pages.codes, pages.scales, pages.table[b:b + 1]
        for i in range(m) if rows is None else [i for i in rows if i < m]:
            want, bound = definition(one, f64(q[at + i:at + i + 1]), [n - m + i + 1], [1], scale, q.dtype)
            y = f64(got[at + i:at + i + 1])
            # what lies beyond 65520 rounds to an infinity in binary16, what may lie on either side of it may be either
            over = np.abs(want) - 65520 if q.dtype == torch.float16 else np.full_like(want, -1e300)
            assert np.array_equal(y[over > bound], np.sign(want[over > bound]) * np.inf), (b, i)
            near = over < -bound
            off = np.abs(y[near] - want[near]) / bound[near]
            assert np.all(np.isfinite(y[near])) and np.all(off <= 1.0 + UNIT[q.dtype]), (b, i, float(off.max()))
        at += m
    return got


def with_scales(lens, hkv, d, page, of_pages, seed):
    """Pages whose values have the scales of_pages[sequence][page of it]; those that do not count are NaN."""
    pages = Pages(lens, hkv, d, page, seed)
    pages.scales[1][:] = float("nan")
    for b, scales in enumerate(of_pages):
        for i in range(-(-lens[b] // page)):
            pages.scales[1][int(pages.table[b, i])] = float(np.float32(scales[i]))
    return pages


@pytest.mark.parametrize("hq,hkv,d,new,most", [(4, 2, 128, 3, 0), (40, 2, 64, 3, 0), (4, 2, 128, 3, 3), (4, 4, 64, 3, 16), (4, 4, 64, 140, 0), (4, 2, 128, 8, 8), (4, 4, 64, 5, 5)])
@pytest.mark.parametrize("page", [16, 64])
def test_values_with_scales_at_the_ends_of_the_range(api, page, hq, hkv, d, new, most):
    """Pages of V that are below 2^-120 (zeros), just above it, or up to 2^240 above or below the others, in every order."""
    n = 12 * page + 3
    scales = [[2.0 ** -126] * 13, [1e-38, 1.0] + [1e-38] * 11, [1.0] * 6 + [2.0 ** -119] * 7, [2.0 ** -119] * 6 + [1.0] * 7, [3e4] * 8 + [1e-36] * 5,
              [2.0 ** (16 * (6 - i)) for i in range(13)], [2.0 ** (16 * (i - 6)) for i in range(13)], [1.0, 0.0, 2.0 ** -100, 0.0] * 3 + [1.0],
              [2.0 ** 100] * 3 + [2.0 ** -100] * 10, [2.0 ** 100] + [2.0 ** -119] * 12, [2.0 ** 119, 2.0 ** -119] * 6 + [1.0], [2.0 ** 60] * 5 + [2.0 ** -20, 2.0 ** 60] * 4]
    lens = [n] * len(scales)
    pages = with_scales(lens, hkv, d, page, scales, 5)
    q = queries(new * len(lens), hq, d, torch.bfloat16, hq)
    got = check_what_is_attended_to(api, pages, q, lens, [new] * len(lens), most, rows=sorted({0, new // 2, new - 1}))
    assert bool(torch.isfinite(got.float()).all()) and not got[:new].any()


@pytest.mark.parametrize("hq,hkv,d,page,new,most", [(4, 4, 64, 16, 120, 0), (4, 4, 128, 16, 300, 0), (8, 2, 64, 16, 30, 0), (40, 2, 128, 32, 40, 0), (1, 1, 128, 64, 200, 0),
                                                    (4, 4, 64, 16, 16, 16), (8, 2, 128, 16, 4, 4), (3, 3, 64, 32, 5, 5), (4, 2, 128, 64, 8, 8)])
@pytest.mark.parametrize("held,late", [(-5, 119), (-119, 120), (3, 40), (0, -119), (100, -119)])
def test_later_pages_have_no_influence(api, held, late, hq, hkv, d, page, new, most):
    """Pages of later tokens whose values are larger or smaller by any factor do not change what earlier tokens see."""
    border = 4 * page if page == 16 else 2 * page  # a page's first token, the middle of the new ones
    n = border - new // 2 + new if border > new // 2 else new
    border = n - new + new // 2 if border <= new // 2 else border
    border -= border % page
    lens = [n, n + 16 * page]
    for dtype in TYPES:
        of_pages = [[2.0 ** (late if i * page >= border + shift else held) for i in range(-(-m // page))] for m, shift in zip(lens, (0, 16 * page))]
        pages = with_scales(lens, hkv, d, page, of_pages, 19)
        q = queries(2 * new, hq, d, dtype, 23)
        rows = sorted({0, new // 4, new // 2 - 1, new // 2, new - 1, max(new // 2 - page, 0), min(new // 2 + page, new - 1)})
        check_what_is_attended_to(api, pages, q, lens, [new, new], most, rows=rows)


@pytest.mark.parametrize("hq,hkv,d,page,new,most", [(4, 4, 64, 16, 250, 0), (16, 2, 128, 16, 16, 0), (40, 2, 64, 32, 50, 0), (2, 2, 128, 16, 16, 16), (1, 1, 64, 16, 700, 0)])
def test_every_token_sees_its_own_pages_only(api, hq, hkv, d, page, new, most):
    """Scales at random over the whole range, among the held tokens' pages too."""
    for seed in range(3):
        rng = np.random.default_rng(seed)
        lens, pieces = [new + 30 + 16 * seed, new + 900], [new, new]
        of_pages = [2.0 ** rng.uniform(-119, 119, -(-n // page)) for n in lens]
        if seed == 2:  # the further on the larger, so that what a token sees of the last page is not lost beside others
            of_pages = [np.sort(x) for x in of_pages]
        pages = with_scales(lens, hkv, d, page, of_pages, 29 + seed)
        q = queries(2 * new, hq, d, torch.bfloat16, 31, 0.3)
        check_what_is_attended_to(api, pages, q, lens, pieces, most, rows=range(0, new, 1 if new <= 16 else 13))


@pytest.mark.parametrize("hq,hkv,d,new,most", [(4, 2, 64, 3, 0), (4, 4, 128, 140, 0), (4, 2, 64, 3, 3)])
def test_values_next_to_the_largest_number(api, hq, hkv, d, new, most):
    """Scales of nearly 2^128 with codes of -1, 0 and 1: the outputs are numbers that bfloat16 has."""
    page = 32
    scales = [[1.98 * 2.0 ** 127] * 13, [1.0, 1.98 * 2.0 ** 127, 2.0 ** 126] * 4 + [1.0], [2.0 ** 100] * 4 + [1.5 * 2.0 ** 127] * 9]
    lens = [12 * page + 3] * 3
    pages = with_scales(lens, hkv, d, page, scales, 37)
    pages.codes[1].copy_(pages.codes[1] % 3 - 1)
    q = queries(new * 3, hq, d, torch.bfloat16, 41, 2.0)
    got = check_what_is_attended_to(api, pages, q, lens, [new] * 3, most, rows=sorted({0, new // 2, new - 1}))
    assert bool(torch.isfinite(got.float()).all())


@pytest.mark.parametrize("hq,hkv,d,new,held", [(1, 1, 128, 240, 80), (4, 4, 64, 100, 70), (40, 2, 64, 3, 127), (10, 2, 128, 60, 100)])
@pytest.mark.parametrize("small,large", [(-100, 100), (100, -100), (-10, 119)])
def test_zeros_between_pages_of_very_different_scales(api, small, large, hq, hkv, d, new, held):
    """Rows whose last tiles hold zeros, with pages behind them that they do not attend to: a reference moves for four tiles at a time."""
    page = 128
    for zeros in (1, 2, 3):
        first = 512 + held  # the first new token, in a tile of zeros
        n = first + new
        of_pages = [2.0 ** small] * 4 + [0.0] * zeros + [2.0 ** large] * 8
        pages = with_scales([n, n + 128], hkv, d, page, [of_pages, [2.0 ** small] * 5 + of_pages[4:]], 43)
        q = queries(2 * new, hq, d, torch.bfloat16, 47)
        check_what_is_attended_to(api, pages, q, [n, n + 128], [new, new], rows=sorted({0, 1, new // 3, new // 2, new - 1}))


@pytest.mark.parametrize("hq,hkv,d,new", [(6, 2, 64, 9), (40, 2, 128, 3), (4, 4, 64, 150)])
@pytest.mark.parametrize("first", [2.0 ** -60, 0.0])
def test_weights_count_in_parts_whose_values_vanish(api, first, hq, hkv, d, new):
    """The first page has all the weight and tiny values or none, the others, up to 2^170 larger, hardly any: units of every length, cut anywhere."""
    page = 64
    for held in range(300, 2200, 173):
        n = held + new
        of_pages = [first, 0.0, 0.0] + [2.0 ** -32, 2.0 ** 110, 2.0 ** -30, 2.0 ** 79] * (n // page)
        pages = with_scales([n, 3], hkv, d, page, [of_pages, [1.0]], 53)
        pages.codes[0][..., 0] = -64
        pages.codes[0][int(pages.table[0, 0]), ..., 0] = 64
        q = 0.05 * queries(new + 2, hq, d, torch.float32, 59)
        q[..., 0] = 150.0
        check_what_is_attended_to(api, pages, q.bfloat16(), [n, 3], [new, 2], 0, 0.2, rows=sorted({0, new // 2, new - 1}))
