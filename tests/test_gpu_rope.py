"""Rotary positions on the GPU (pd_rope, pd_kv_append_rope) against fp64 definitions.

Bound of a turned value, with x and y the pair's values: the angle is rounded to binary32 as a part of half a turn (2^-25 of pi at most), its
sine and cosine are off by 2 units in the last place at most (2^-23), the two products and their sum are rounded (2^-24 each): below 2^-21
(|x| + |y|) in all; positions up to 2^24, whose products with a frequency binary64 holds exactly.  Then one rounding to the type,
u = 2^-11 or 2^-8 relative and half its smallest step.  Codes: half a step, three binary32 roundings of numbers up to 127 (2.3e-5 steps), the
turned value's own error, and that of the page's scale, which is as large relative to the page's largest value."""
import numpy as np
import pytest
import torch

from oracle import pd_oracle_attn as orc

pytestmark = pytest.mark.gpu
UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
SMALLEST = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
TYPES = [torch.float16, torch.bfloat16]
TURN = 2.0 ** -21


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2512_19720_b200 import api
    return api


def f64(t):
    return t.detach().cpu().double().numpy()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def offsets(lens):
    return i32(np.concatenate([[0], np.cumsum(lens)]).tolist())


def frequencies(pairs, base=10000.0):
    return (base ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float().cuda()


def partner(x, pairs, interleaved):
    """|x| + |y| of each value's pair; 0 where nothing turns."""
    out = np.zeros_like(x)
    first = np.arange(pairs) * 2 if interleaved else np.arange(pairs)
    second = first + (1 if interleaved else pairs)
    out[..., first] = out[..., second] = np.abs(x[..., first]) + np.abs(x[..., second])
    return out


def check_turned(got, x, positions, inv_freq, axes, interleaved, inverse=False):
    x, pairs = f64(x), inv_freq.numel()
    axes = [0] * pairs if axes is None else axes.tolist()
    want = orc.rope(x, np.atleast_2d(f64(positions)), f64(inv_freq), axes, interleaved, inverse)
    bound = (UNIT[got.dtype] + 2.0 ** -30) * np.abs(want) + SMALLEST[got.dtype] + TURN * partner(x, pairs, interleaved)
    assert np.all(np.abs(f64(got) - want) <= bound), float((np.abs(f64(got) - want) / bound).max())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hk,d,pairs", [(8, 2, 128, 64), (5, 5, 64, 32), (3, 1, 128, 48), (40, 8, 128, 8), (64, 8, 128, 64), (7, 0, 64, 24), (1, 1, 64, 8), (64, 64, 64, 32)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n_axes", [1, 3])
def test_rope_matches_the_definition(api, hq, hk, d, pairs, interleaved, n_axes, dtype):
    t = 13
    gen = torch.Generator("cuda").manual_seed(hq + pairs)
    qk = torch.randn(t, hq + hk, d, generator=gen, device="cuda").to(dtype)
    q, k = qk[:, :hq], qk[:, hq:] if hk else None
    positions = torch.randint(0, 1 << 20, (n_axes, t), generator=gen, device="cuda", dtype=torch.int32)
    positions[0, :4] = i32([0, 1, -5, 131071])
    axes = None if n_axes == 1 else torch.randint(0, n_axes, (pairs,), generator=gen, device="cuda", dtype=torch.int32)
    inv_freq = frequencies(pairs)
    q1, k1 = api.pd_rope(q, k, positions, inv_freq, axes, interleaved)
    assert api.pd_device_status(api.attn_workspace()) == 0
    check_turned(q1, q, positions, inv_freq, axes, interleaved)
    if hk:
        check_turned(k1, k, positions, inv_freq, axes, interleaved)
    # in place, and into the middle of wider tensors; back again
    whole = qk.clone()
    api.pd_rope(whole[:, :hq], whole[:, hq:] if hk else None, positions, inv_freq, axes, interleaved, q_out=whole[:, :hq], k_out=whole[:, hq:] if hk else None)
    assert torch.equal(whole[:, :hq], q1) and (hk == 0 or torch.equal(whole[:, hq:], k1))
    wide = torch.full((t, hq + 2, d + 16), 7.0, dtype=dtype, device="cuda")
    api.pd_rope(q, None, positions, inv_freq, axes, interleaved, q_out=wide[:, 1:hq + 1, 8:d + 8])
    assert torch.equal(wide[:, 1:hq + 1, 8:d + 8], q1)
    wide[:, 1:hq + 1, 8:d + 8] = 7.0
    assert bool((wide == 7.0).all())
    back, _ = api.pd_rope(q1, None, positions, inv_freq, axes, interleaved, inverse=True)
    check_turned(back, q1, positions, inv_freq, axes, interleaved, inverse=True)
    if 2 * pairs < d:
        assert torch.equal(q1[..., 2 * pairs:], q[..., 2 * pairs:])


def test_rope_gradient(api):
    """The inverse is the gradient's way: sum(g . rope(x)) against differences along random directions; the map is linear, so that a
    difference has no error but the roundings: 2 u |g| |direction| summed over the values."""
    t, h, d, pairs = 9, 4, 64, 32
    gen = torch.Generator("cuda").manual_seed(5)
    x, g, e = (torch.randn(t, h, d, generator=gen, device="cuda").half() for _ in range(3))
    positions, inv_freq = torch.arange(t, device="cuda", dtype=torch.int32) * 37, frequencies(pairs)
    grad, _ = api.pd_rope(g, None, positions, inv_freq, inverse=True)
    up, _ = api.pd_rope((x + e), None, positions, inv_freq)
    down, _ = api.pd_rope((x - e), None, positions, inv_freq)
    moved = (x + e).double() - (x - e).double()  # what the roundings of x + e and x - e left
    want = (g.double() * (up.double() - down.double())).sum()
    got = (grad.double() * moved).sum()
    room = 2.0 ** -11 * ((g.double().abs() * (up.double().abs() + down.double().abs())).sum() + (grad.double().abs() * moved.abs()).sum()) * 1.01
    assert abs(float(want - got)) <= float(room)


def test_rope_many_tokens_far_positions_and_strides(api):
    t, hq, hk, d, pairs = 3000, 6, 3, 128, 64
    gen = torch.Generator("cuda").manual_seed(9)
    q = torch.randn(hq, t, d, generator=gen, device="cuda").bfloat16().transpose(0, 1)  # heads before tokens
    k = torch.randn(t, hk, d, generator=gen, device="cuda").bfloat16()
    rows = torch.randint(0, 1 << 24, (3, t + 50), generator=gen, device="cuda", dtype=torch.int32)
    positions = rows[:, 20:t + 20]  # rows further apart than they are long
    axes, inv_freq = i32([0, 1, 2, 1] * 16), frequencies(pairs, 500000.0)
    q1, k1 = api.pd_rope(q, k, positions, inv_freq, axes)
    at = torch.randint(0, t, (40,), generator=gen, device="cuda")
    check_turned(q1[at], q[at], positions[:, at], inv_freq, axes, False)
    check_turned(k1[at], k[at], positions[:, at], inv_freq, axes, False)


def test_rope_bad_axes_are_reported(api):
    q = torch.randn(4, 2, 64, device="cuda").half()
    positions, inv_freq = torch.ones(2, 4, dtype=torch.int32, device="cuda"), frequencies(32)
    good, _ = api.pd_rope(q, None, positions, inv_freq, i32([0, 1] * 16))
    for bad in (-1, 2, 2 ** 31 - 1):
        axes = i32([0, 1] * 16)
        axes[3] = bad
        got, _ = api.pd_rope(q, None, positions, inv_freq, axes)
        assert api.pd_device_status(api.attn_workspace()) == 8
        assert torch.equal(got, good)  # all axes hold the same here
    assert api.pd_rope(q[:0], None, positions[:, :0], inv_freq, i32([0, 1] * 16))[0].shape == (0, 2, 64)


# ------------------------------------------------------------------ appending
class Pages:
    """A cache with its pages in random order; unused pages and table entries hold what must not be looked at."""

    def __init__(self, lens, hkv, d, page, seed, extra=3):
        rng = np.random.default_rng(seed)
        self.page, n = page, [-(-x // page) for x in lens]
        order = rng.permutation(sum(n) + extra)
        self.table = np.full((len(lens), max(max(n), 1) + 2), -7, dtype=np.int64)
        at = 0
        for b, m in enumerate(n):
            self.table[b, :m] = order[at:at + m]
            at += m
        shape = (sum(n) + extra, hkv, page, d)
        self.codes = [torch.from_numpy(rng.integers(-127, 128, shape).astype(np.int8)).cuda() for _ in range(2)]
        self.scales = [torch.from_numpy(np.exp(rng.normal(-4, 1.0, shape[:2])).astype(np.float32)).cuda() for _ in range(2)]
        for s in self.scales:
            s[torch.from_numpy(order[at:]).cuda()] = float("nan")
        self.block_table = i32(self.table.tolist())

    def tensors(self):
        return *self.codes, *self.scales


def check_append(api, held, new, hq, hkv, d, page, pairs, dtype, seed, n_axes=1, interleaved=False, amplitude=1.0, given=True):
    total, t = [a + b for a, b in zip(held, new)], sum(new)
    pages = Pages(total, hkv, d, page, seed)
    gen = torch.Generator("cuda").manual_seed(seed)
    qkv = (amplitude * torch.randn(t, hq + 2 * hkv, d, generator=gen, device="cuda")).to(dtype)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    inv_freq = frequencies(pairs)
    axes = None if n_axes == 1 else torch.randint(0, n_axes, (pairs,), generator=gen, device="cuda", dtype=torch.int32)
    place = np.concatenate([np.arange(h, h + m) for h, m in zip(held, new)])
    positions = torch.randint(0, 100000, (n_axes, t), generator=gen, device="cuda", dtype=torch.int32) if given else i32([place.tolist()])
    before = [x.cpu().numpy() for x in pages.tensors()]
    out = [torch.full((t, hkv, d), 9.0, dtype=dtype, device="cuda") for _ in range(2)]
    q1 = api.pd_kv_append_rope(q if hq else None, k, v, *pages.tensors(), offsets(new), i32(total), pages.block_table, inv_freq, positions if given else None, axes,
                               interleaved, k_values=out[0], v_values=out[1])
    assert api.pd_device_status(api.attn_workspace()) == 0
    if hq:
        check_turned(q1, q, positions, inv_freq, axes, interleaved)
    after = [x.cpu().numpy() for x in pages.tensors()]
    turned = orc.rope(f64(k), f64(positions), f64(inv_freq), [0] * pairs if axes is None else axes.tolist(), interleaved)
    for which, x, slack in ((0, turned, TURN * partner(f64(k), pairs, interleaved)), (1, f64(v), np.zeros_like(turned))):
        codes0, scale0, codes1, scale1, values = before[which], before[2 + which], after[which], after[2 + which], f64(out[which])
        slots, fresh, at = np.zeros((codes0.shape[0], page), dtype=bool), np.zeros(scale0.shape[0], dtype=bool), 0
        for b, (h, m) in enumerate(zip(held, new)):
            for p0 in range(h // page * page, h + m if m else 0, page):
                p, lo, hi = pages.table[b][p0 // page], max(h, p0), min(h + m, p0 + page)
                part, loose = x[at + lo - h:at + hi - h], slack[at + lo - h:at + hi - h]
                most = np.abs(part).max(axis=(0, 2))
                s_old = np.zeros(hkv) if lo == p0 else scale0[p].astype(np.float64)
                want = np.maximum(s_old, most / 127)
                assert np.all(np.abs(scale1[p] - want) <= 2.0 ** -23 * want + loose.max(axis=(0, 2)) / 127 * 1.01), (b, p0)
                fresh[p] = True
                step = scale1[p].astype(np.float64)[:, None]
                slots[p, :hi - p0] = True
                old = codes0[p, :, :lo - p0].astype(np.float64) * scale0[p].astype(np.float64)[:, None, None]
                assert np.all(np.abs(codes1[p, :, :lo - p0] * step[:, None] - old) <= (0.5 + 2.3e-5) * step[:, None])
                for i in range(hi - lo):
                    got = codes1[p, :, lo - p0 + i].astype(np.float64) * step
                    assert np.all(np.abs(got - part[i]) <= (0.5 + 2.3e-5) * step + loose[i]), (b, lo + i)
                    val = values[at + lo - h + i]
                    assert np.all(np.abs(val - got) <= (UNIT[dtype] + 2.0 ** -22) * np.abs(val) + SMALLEST[dtype])
            at += m
        where = np.broadcast_to(~slots[:, None, :, None], codes1.shape)
        assert np.array_equal(codes1[where], codes0[where])  # nothing else is written
        assert np.array_equal(scale1[~fresh], scale0[~fresh], equal_nan=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hkv,d,page,pairs", [(4, 2, 128, 64, 64), (3, 1, 64, 16, 32), (6, 3, 64, 128, 24), (0, 2, 128, 128, 64), (16, 2, 128, 16, 48), (5, 5, 64, 32, 8),
                                                 (12, 12, 128, 32, 64), (18, 9, 64, 64, 32)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_matches_the_definition(api, hq, hkv, d, page, pairs, interleaved, dtype):
    """Pieces of one token to several pages, on both sides of the length that the two kinds of blocks take, with pages gone on with."""
    held = [0, 5, page - 1, page, 3 * page + 2, 17, 0, page - 3, page - 4]
    new = [2 * page + 3, page, 1, 1, 0, 2 * page, 1, 8, 9]
    check_append(api, held, new, hq, hkv, d, page, pairs, dtype, 67, 1 if interleaved else 3, interleaved)


@pytest.mark.parametrize("new", [[1] * 300, [1, 2, 8, 3] * 20, [0, 9, 0, 30], [7], [8], [9], [1]], ids=lambda x: f"{len(x)}x{x[0]}")
def test_append_places_in_sequences(api, new):
    """Without positions; growing and staying scales."""
    rng = np.random.default_rng(71)
    for amplitude in (0.01, 1.0, 100.0):
        check_append(api, rng.integers(0, 70, len(new)).tolist(), new, 4, 2, 64, 32, 32, torch.float16, 73, amplitude=amplitude, given=False)


def test_append_is_rotation_and_append(api):
    """Where nothing turns (all positions 0) the calls are pd_kv_append's, bit for bit; so are values at any positions."""
    held, new, hkv, d, page = [0, 100, 33], [150, 1, 40], 2, 128, 64
    total = [a + b for a, b in zip(held, new)]
    one, two = Pages(total, hkv, d, page, 3), Pages(total, hkv, d, page, 3)
    k, v = (torch.randn(sum(new), hkv, d, generator=torch.Generator("cuda").manual_seed(i), device="cuda").half() for i in range(2))
    api.pd_kv_append(k, v, *one.tensors(), offsets(new), i32(total), one.block_table)
    api.pd_kv_append_rope(None, k, v, *two.tensors(), offsets(new), i32(total), two.block_table, frequencies(64), torch.zeros(sum(new), dtype=torch.int32, device="cuda"))
    assert all(torch.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(one.tensors(), two.tensors()))
    two = Pages(total, hkv, d, page, 3)
    api.pd_kv_append_rope(None, k, v, *two.tensors(), offsets(new), i32(total), two.block_table, frequencies(64))
    assert torch.equal(one.codes[1], two.codes[1]) and not torch.equal(one.codes[0], two.codes[0])


def test_append_rows_of_no_sequence_and_values_in_place(api):
    hkv, d, page, t = 2, 64, 32, 60
    gen = torch.Generator("cuda").manual_seed(11)
    q, k, v = (torch.randn(t, hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(3))
    fresh = lambda: [torch.zeros(4, hkv, page, d, dtype=torch.int8, device="cuda") for _ in range(2)] + [torch.zeros(4, hkv, device="cuda") for _ in range(2)]  # noqa: E731
    cu, lens, table = i32([3, 50, 50, 52]), i32([47, 0, 2]), i32([[1, 3], [-1, -1], [0, -1]])
    one, two, three = fresh(), fresh(), fresh()
    q1 = torch.full_like(q, 7.0)
    values = [torch.full_like(k, 7.0) for _ in range(2)]
    api.pd_kv_append_rope(q, k, v, *one, cu, lens, table, frequencies(32), q_out=q1, k_values=values[0], v_values=values[1])
    for x in (q1, *values):
        assert bool((x[:3] == 7.0).all() and (x[52:] == 7.0).all() and (x[3:52] != 7.0).any())
    q2, k2, v2 = q.clone(), k.clone(), v.clone()
    assert api.pd_kv_append_rope(q2, k2, v2, *two, cu, lens, table, frequencies(32), q_out=q2, k_values=k2, v_values=v2).data_ptr() == q2.data_ptr()
    assert torch.equal(q2[3:52], q1[3:52]) and torch.equal(k2[3:52], values[0][3:52]) and torch.equal(v2[3:52], values[1][3:52]) and torch.equal(q2[52:], q[52:])
    api.pd_kv_append_rope(None, k, v, *three, cu, lens, table, frequencies(32))
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(one, two, three))
    assert api.pd_device_status(api.attn_workspace()) == 0


def test_append_bad_indices_are_reported(api):
    hkv, d, page = 2, 128, 32
    q, k, v = (torch.randn(50, hkv, d, device="cuda").half() for _ in range(3))
    for cu, lens, tab in (([0, 51], [51], [[1, 3]]), ([0, 50], [49], [[1, 3]]), ([0, 50], [50], [[1, 4]]), ([0, 50], [50], [[-1, 3]]), ([0, 50], [70], [[1, 3]]),
                          ([0, 5], [4], [[1, 3]]), ([0, 5], [5], [[4, 3]]), ([0, 5], [69], [[1, 3]]), ([9, 5], [5], [[1, 3]]), ([-1, 5], [6], [[1, 3]])):
        guard = [torch.full((6, hkv, page, d), 99, dtype=torch.int8, device="cuda") for _ in range(2)] + [torch.full((6, hkv), 3.0, device="cuda") for _ in range(2)]
        cache = [g[1:5] for g in guard]
        api.pd_kv_append_rope(q, k, v, *cache, i32(cu), i32(lens), i32(tab), frequencies(64))
        assert api.pd_device_status(api.attn_workspace()) == 8, (cu, lens, tab)
        assert all(bool((g[0] == g[5]).all()) and float(g[0].flatten()[0]) in (99, 3) for g in guard)
    assert api.pd_device_status(api.attn_workspace()) == 0


def test_append_zeros_tiny_and_non_finite_values(api):
    page, d = 16, 64
    for new in ([40], [8] * 5):  # both kinds of blocks
        for dtype in TYPES:
            codes = [torch.full((8, 1, page, d), 99, dtype=torch.int8, device="cuda") for _ in range(2)]
            scales = [torch.full((8, 1), 3.0, device="cuda") for _ in range(2)]
            k, v = torch.zeros(40, 1, d, dtype=dtype, device="cuda"), torch.ones(40, 1, d, dtype=dtype, device="cuda")
            if dtype == torch.bfloat16:
                k[16:32] = 1e-38  # a scale below 2^-120
            v[20, 0, 3], v[35, 0, 4] = float("inf"), float("nan")
            k[33, 0, 7] = float("nan")
            values = [torch.empty_like(k) for _ in range(2)]
            table = i32([[2, 0, 3]]) if len(new) == 1 else i32([[2], [0], [3], [5], [6]])
            api.pd_kv_append_rope(None, k, v, *codes, *scales, offsets(new), i32(new), table, frequencies(32), k_values=values[0], v_values=values[1])
            assert not codes[0][2, :, :8].any() and not codes[0][0, :, :8].any() and not values[0].float()[:16].any() and float(scales[0][2]) == 0.0
            assert bool((codes[0][1] == 99).all()) and float(scales[0][1]) == 3.0 and bool((values[1][:16] == 1).all())
            inf_page, nan_page = (0, 3) if len(new) == 1 else (3, 6)
            assert bool(torch.isinf(scales[1][inf_page]).all()) and bool(torch.isnan(scales[1][nan_page]).all()) and bool(torch.isnan(scales[0][nan_page]).all())
            assert not codes[1][inf_page, :, :8].any() and not codes[1][nan_page, :, :8].any() and not codes[0][nan_page, :, :8].any()  # the slots that hold tokens
