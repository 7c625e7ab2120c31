"""Paths of pd_kv_append_rope and pd_rope that only larger calls take: walks of a block over several heads, pages found by tokens, queries in
a launch of their own; and positions at the ends of their range.  Bounds are those of test_gpu_rope."""
import numpy as np
import pytest
import torch

from test_gpu_rope import SMALLEST, TURN, TYPES, UNIT, check_append, check_turned, f64, frequencies, i32, offsets, partner

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2512_19720_b200 import api
    return api


@pytest.mark.parametrize("held,new,hq,hkv,d,page,pairs", [
    ([0, 30, 64, 1], [512, 500, 300, 700], 2, 32, 128, 64, 64),   # a head a round, four or more rounds
    ([7, 0], [2400, 2500], 0, 7, 128, 16, 64),                    # four heads a round, the last round with three
    ([0, 127], [700, 1300], 6, 24, 128, 128, 64),                 # blocks of 512 threads
    ([128, 3, 5], [129, 8, 140], 4, 3, 128, 128, 32),             # the same, queries in the same launch, both kinds of sequences
    ([5, 0], [1900, 31], 3, 20, 64, 32, 8)], ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
def test_blocks_that_walk_over_heads(api, held, new, hq, hkv, d, page, pairs, interleaved):
    check_append(api, held, new, hq, hkv, d, page, pairs, TYPES[interleaved], 101, 3, interleaved)


@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("given", [False, True])
def test_few_long_pieces_among_many_sequences(api, page, given):
    """Fewer than nine new tokens a sequence on average: pages are told apart by tokens.  Long pieces behind none, single ones and each other."""
    new = [1] * 60 + [9, 9, 0, 40, 300, 1, 0, 9] + [0] * 50 + [1, 8, 17, 9] + [1, 0, 0] * 20 + [40, 10, 9]
    rng = np.random.default_rng(5)
    held = rng.integers(0, 3 * page, len(new)).tolist()
    for b in (60, 67, len(new) - 1):  # nine tokens across a page's border
        held[b] = page - 4
    assert sum(new) < 9 * len(new)
    check_append(api, held, new, 2, 2, 64, page, 32, torch.float16, 103, given=given)
    check_append(api, held, new, 3, 3, 128, page, 48, torch.bfloat16, 107, 2, True)


@pytest.mark.parametrize("interleaved,given", [(False, True), (True, False)])
def test_many_queries(api, interleaved, given):
    """Queries in a launch of their own, in place as well: the rotation's bits, and rows of no sequence left as they are."""
    hq, d, page, pairs = 64, 128, 64, 64
    new, t = [2000, 0, 5, 2300], 4400
    held = [10, 0, 60, 0]
    first = 20
    gen = torch.Generator("cuda").manual_seed(7)
    q, k, v = (torch.randn(t, h, d, generator=gen, device="cuda").to(TYPES[interleaved]) for h in (hq, 1, 1))
    assert t * hq * d >= 1 << 25
    cu = offsets(new) + first
    lens = [a + b for a, b in zip(held, new)]
    n = [-(-x // page) for x in lens]
    table = i32([[sum(n[:b]) + i if i < n[b] else -1 for i in range(max(n))] for b in range(4)])
    cache = [torch.zeros(sum(n), 1, page, d, dtype=torch.int8, device="cuda") for _ in range(2)] + [torch.ones(sum(n), 1, device="cuda") for _ in range(2)]
    place = np.zeros(t, dtype=np.int64)
    place[first:first + sum(new)] = np.concatenate([np.arange(h, h + m) for h, m in zip(held, new)])
    positions = i32((place * 3 + 1 if given else place).tolist())
    out = torch.full_like(q, 7.0)
    freq = frequencies(pairs)
    api.pd_kv_append_rope(q, k, v, *cache, cu, i32(lens), table, freq, positions if given else None, None, interleaved, q_out=out)
    assert api.pd_device_status(api.attn_workspace()) == 0
    last = first + sum(new)
    assert bool((out[:first] == 7.0).all() and (out[last:] == 7.0).all())
    some = torch.randint(first, last, (30,), generator=gen, device="cuda")
    check_turned(out[some], q[some], positions[some], freq, None, interleaved)
    turned, _ = api.pd_rope(q, None, positions, freq, None, interleaved)
    assert torch.equal(out[first:last], turned[first:last])
    again = q.clone()
    api.pd_kv_append_rope(again, k, v, *cache, cu, i32(lens), table, freq, positions if given else None, None, interleaved, q_out=again)
    assert torch.equal(again[first:last], turned[first:last]) and torch.equal(again[:first], q[:first]) and torch.equal(again[last:], q[last:])


@pytest.mark.parametrize("interleaved", [False, True])
def test_positions_at_the_ends_of_their_range(api, interleaved):
    """The angle a = position * frequency is rounded to binary64 once, its part of a turn by the factor's and the product's rounding: below
    2^-51 |a| in all, beside what test_gpu_rope counts.  The definition in 64-bit significands holds the product exactly."""
    assert np.finfo(np.longdouble).nmant >= 63
    places = [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2, -2 ** 31 + 1, 2 ** 30 + 12345, -2 ** 30 - 54321, 1999999999, 131071, 2 ** 24 + 1, 0]
    d, h = 64, 3
    freq = frequencies(32)
    freq[3], freq[5] = 0.9999999, 1.9999999
    angles = np.array(places, dtype=np.longdouble)[:, None] * f64(freq).astype(np.longdouble)[None]
    two_pi = np.longdouble("6.283185307179586476925286766559")
    part = np.remainder(angles, two_pi).astype(np.float64)
    for dtype in TYPES:
        q = torch.randn(len(places), h, d, generator=torch.Generator("cuda").manual_seed(3), device="cuda").to(dtype)
        x = f64(q)
        a, b = (slice(0, 64, 2), slice(1, 64, 2)) if interleaved else (slice(0, 32), slice(32, 64))
        loose = np.zeros_like(x)
        loose[..., a] = loose[..., b] = np.abs(angles).astype(np.float64)[:, None] * 2.0 ** -51
        for inverse in (False, True):
            c, s = np.cos(part)[:, None], np.sin(part)[:, None] * (-1 if inverse else 1)
            want = np.zeros_like(x)
            want[..., a], want[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
            got, _ = api.pd_rope(q, None, i32(places), freq, None, interleaved, inverse)
            bound = (UNIT[dtype] + 2.0 ** -30) * np.abs(want) + SMALLEST[dtype] + (TURN + loose) * partner(x, 32, interleaved)
            assert np.all(np.abs(f64(got) - want) <= bound), float((np.abs(f64(got) - want) / bound).max())
