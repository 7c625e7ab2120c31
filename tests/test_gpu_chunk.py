"""Attention of pieces over the 8-bit cache on the GPU (pd_attn_chunk) against fp64 definitions.

Bound of an output, with w_j the weights and M the largest score of the row, L = sum_j e^(s_j - M):
  - rounding to the output's type: u_out |out| (2^-11 or 2^-8), and its smallest step;
  - P in binary16: 2^-11 sum_j w_j |v_j|, and 2^-17 of it for exponentials and the logarithm of a page's scale in binary32; where P is
    subnormal 2^-25 of a unit of 2^-7 r, r at most 2^7 times the page's scale: at most |v_j| 2^-24 / L, and never more than the weight itself;
  - scores: products are exact, their sums off by at most 2^-19 of sum |q| |k|, further arithmetic by 2^-20 (|s_j| + 1).  Weights are off
    by e^(2 max d) - 1 then;
  - pages whose scale is below 2^-60 of the sequence's largest: 2^-60 of the largest |v_j|."""
import numpy as np
import pytest
import torch

from oracle import pd_oracle_attn as orc
from test_gpu_rope import Pages, frequencies, i32, offsets

pytestmark = pytest.mark.gpu
UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
SMALLEST = {torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}
TYPES = [torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2512_19720_b200 import api
    return api


def f64(t):
    return t.detach().cpu().double().numpy()


def definition(pages, q, lens, new, scale, dtype, only=None):
    """Outputs and their bound for queries q (fp64) [T, Hq, d]; `only`: rows of interest."""
    out, bound, at = np.zeros_like(q), np.zeros_like(q), 0
    kc, vc, ks, vs = (x.cpu().numpy().astype(np.float64) for x in pages.tensors())
    ks, vs = np.where(ks < 2.0 ** -120, 0, ks), np.where(vs < 2.0 ** -120, 0, vs)
    group = q.shape[1] // kc.shape[1]
    for b, (n, m) in enumerate(zip(lens, new)):
        p = pages.table[b][:-(-n // pages.page)]
        rows = [i for i in range(m) if only is None or at + i in only]
        for g in range(kc.shape[1] if rows else 0):
            k = (kc[p, g] * ks[p, g][:, None, None]).reshape(-1, q.shape[2])[:n]
            v = (vc[p, g] * vs[p, g][:, None, None]).reshape(-1, q.shape[2])[:n]
            for h in range(g * group, (g + 1) * group):
                x = q[[at + i for i in rows], h]
                s = x @ k.T * scale
                off = abs(scale) * 2.0 ** -19 * (np.abs(x) @ np.abs(k).T) + 2.0 ** -20 * (np.abs(s) + 1)
                hidden = np.arange(n)[None, :] > np.array(rows)[:, None] + n - m
                s[hidden], off[hidden] = -np.inf, 0.0
                e = np.exp(s - s.max(1, keepdims=True))
                total = e.sum(1, keepdims=True)
                w, spread = e / total, np.expm1(2 * off.max(1, keepdims=True))
                o = w @ v
                out[[at + i for i in rows], h] = o
                most = np.abs(v).max()
                bound[[at + i for i in rows], h] = (UNIT[dtype] * np.abs(o) + SMALLEST[dtype] + (2.0 ** -11 + 2.0 ** -17 + spread) * (w @ np.abs(v)) +
                                                    np.minimum(w, 2.0 ** -24 / total) @ np.abs(v) + 2.0 ** -60 * most)
        at += m
    return out, bound


def check(api, pages, q, lens, new, scale=None, got=None, only=None, max_new=0):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    if got is None:
        got = api.pd_attn_chunk(q, *pages.tensors(), offsets(new), i32(lens), pages.block_table, max_new, scale)
        assert api.pd_device_status(api.chunk_workspace()) == 0
    want, bound = definition(pages, f64(q), lens, new, scale, q.dtype, only)
    rows = slice(None) if only is None else sorted(only)
    y, want, bound = f64(got)[rows], want[rows], bound[rows]
    # what lies beyond 65520 rounds to an infinity in binary16, what may lie on either side of it may be either
    over = np.abs(want) - 65520 if q.dtype == torch.float16 else np.full_like(want, -1e300)
    assert np.array_equal(y[over > bound], np.sign(want[over > bound]) * np.inf)
    near = over < -bound
    off = np.abs(y[near] - want[near]) / bound[near]
    assert np.all(np.isfinite(y[near])) and off.max() <= 1.0, float(off.max())
    return got


def queries(t, hq, d, dtype, seed, sd=1.0):
    return (sd * torch.randn(t, hq, d, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")).to(dtype)


def test_definition_against_single_tokens():
    """The vectorised definition above is that of the oracle, row by row."""
    pages = Pages([9, 40], 2, 64, 16, 3)
    q = queries(9, 4, 64, torch.float16, 1)
    want = orc.attn_chunk(f64(q), *(x.cpu().numpy() for x in pages.tensors()), [9, 40], [9, 0], pages.table, 0.1)
    got, _ = definition(pages, f64(q), [9, 40], [9, 0], 0.1, torch.float16)
    assert np.allclose(got, want, atol=1e-12)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hkv,d,page", [(4, 4, 128, 64), (8, 1, 128, 16), (6, 2, 64, 32), (10, 2, 128, 128), (1, 1, 64, 16)])
@pytest.mark.parametrize("new", [[1], [5], [33], [130], [1, 0, 7, 65, 200]], ids=str)
def test_chunk_matches_the_definition(api, new, hq, hkv, d, page, dtype):
    held = [77, 0, 130, 1, 250][:len(new)]
    lens = [a + b for a, b in zip(held, new)]
    pages = Pages(lens, hkv, d, page, 5 + hq)
    q = queries(sum(new), hq, d, dtype, sum(new))
    for most in (0, max(new)):  # few rows, where the most new tokens are known, go to another kernel
        got = check(api, pages, q, lens, new, max_new=most)
        again = api.pd_attn_chunk(q, *pages.tensors(), offsets(new), i32(lens), pages.block_table, most)
        assert torch.equal(got, again)  # the same bits


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hkv,d,page,most", [(4, 4, 128, 64, 8), (5, 5, 64, 16, 16), (16, 8, 128, 32, 4), (8, 2, 64, 128, 4), (32, 2, 128, 16, 1), (8, 1, 128, 64, 2), (12, 4, 64, 32, 5)])
def test_chunk_few_rows(api, hq, hkv, d, page, most, dtype):
    """At most 16 rows share a key/value head: every number of tokens, none among them, at the ends of pages and tiles, short and long."""
    rng = np.random.default_rng(most)
    new = list(range(most + 1)) + rng.integers(0, most + 1, 20).tolist() + [most, 1]
    held = rng.choice([0, 1, 15, 16, 31, 32, 33, 64, 127, 128, 300], len(new)).tolist()
    held[-2:] = [5000, 3000]
    lens = [a + b for a, b in zip(held, new)]
    pages = Pages(lens, hkv, d, page, 31 + most)
    q = queries(sum(new), hq, d, dtype, 7)
    got = check(api, pages, q, lens, new, max_new=most)
    for _ in range(3):
        assert torch.equal(got, api.pd_attn_chunk(q, *pages.tensors(), offsets(new), i32(lens), pages.block_table, most))
    check(api, pages, q, lens, new, -0.1, max_new=most)


@pytest.mark.parametrize("hq,hkv,d", [(8, 8, 128), (16, 2, 64), (16, 1, 128), (130, 1, 64), (300, 2, 64), (40, 8, 128)])
@pytest.mark.parametrize("held,new", [([0], [300]), ([9000], [3]), ([20011, 0, 5], [1, 700, 16]), ([127, 128, 129], [1, 128, 127])], ids=str)
def test_chunk_split_over_blocks(api, held, new, hq, hkv, d):
    """Few rows or many: the keys of a unit are dealt to several blocks, whose parts are joined."""
    if max(held) > 5000 and hq > 100:
        held = [h // 8 for h in held]
    lens = [a + b for a, b in zip(held, new)]
    pages = Pages(lens, hkv, d, 64, 29)
    rng = np.random.default_rng(1)
    only = set(rng.integers(0, sum(new), 24).tolist()) | {0, sum(new) - 1, new[0] - 1}
    check(api, pages, queries(sum(new), hq, d, torch.float16, 31), lens, new, 0.05, only=only)


def test_chunk_short_units_of_both_kinds_again_and_again(api):
    """Units of one to four tiles, some whose slots hold the same rows and some whose do not, in turn: the same bits every time."""
    for hq, hkv, new, held in ((10, 2, [1, 0, 7, 65, 200], 250), (8, 8, [130, 257, 5, 140], 0), (16, 4, [40, 33, 70, 3, 65] * 4, 60)):
        lens = [n + held for n in new]
        pages = Pages(lens, hkv, 128, 128, 83)
        q = queries(sum(new), hq, 128, torch.bfloat16, 5)
        first = check(api, pages, q, lens, new)
        for _ in range(100):
            assert torch.equal(first, api.pd_attn_chunk(q, *pages.tensors(), offsets(new), i32(lens), pages.block_table))


@pytest.mark.parametrize("dtype", TYPES)
def test_chunk_many_sequences(api, dtype):
    rng = np.random.default_rng(37)
    new = rng.choice([0, 0, 1, 1, 2, 5, 40], 700).tolist()  # more sequences than threads in a block
    lens = [int(n + h) for n, h in zip(new, rng.integers(0, 90, 700))]
    pages = Pages(lens, 2, 64, 16, 41)
    check(api, pages, queries(sum(new), 4, 64, dtype, 1), lens, new, max_new=40)


@pytest.mark.parametrize("scale", [0.15, -0.15, 0.0])
def test_chunk_scales_of_scores(api, scale):
    new, lens = [20, 150], [300, 170]
    for dtype in TYPES:
        pages = Pages(lens, 2, 64, 32, 7)
        check(api, pages, queries(170, 4, 64, dtype, 9, 3.0), lens, new, scale)


def test_chunk_rising_and_falling_scores(api):
    """Keys that make the running maximum grow at every tile, or never; scores that are far from zero."""
    n, d = 1500, 64
    for sign in (1.0, -1.0):
        for size in (1.0, 60.0):
            pages = Pages([n], 1, d, 16, 11)
            pages.codes[0][:] = 1
            for i in range(-(-n // 16)):
                pages.scales[0][pages.table[0, i]] = (100 + sign * i) / 40
            q = queries(140, 2, d, torch.float16, 13).abs() * 0.1 * size
            check(api, pages, q, [n], [140], 0.05)


def test_chunk_scores_of_any_size(api):
    """One-hot softmax rows: the largest score leads by far more than its own rounding, so that the output is that token's value."""
    n, d = 700, 64
    for exponent in (3, 20, 60, 100):
        pages = Pages([n], 1, d, 64, 17)
        pages.codes[0][:] = 0
        for i in range(n):
            pages.codes[0][pages.table[0, i // 64], 0, i % 64] = (i * 37) % 101
        pages.scales[0][:] = 2.0 ** exponent
        q = torch.ones(50, 1, d, device="cuda").bfloat16()
        got = f64(api.pd_attn_chunk(q, *pages.tensors(), offsets([50]), i32([n]), pages.block_table, 0, 1.0))
        for r in range(50):
            order = (np.arange(n - 50 + r + 1) * 37) % 101
            best = np.flatnonzero(order == order.max())
            v = np.mean([f64(pages.codes[1][pages.table[0, i // 64], 0, i % 64]) * float(pages.scales[1][pages.table[0, i // 64], 0]) for i in best], axis=0)
            assert np.all(np.abs(got[r, 0] - v) <= (2.0 ** -8 + 2.0 ** -10) * np.abs(v).max()), (exponent, r)


@pytest.mark.parametrize("hq,hkv,d,page", [(4, 2, 128, 16), (4, 2, 64, 64), (16, 2, 128, 32)])
def test_chunk_values_with_scales_of_any_size(api, hq, hkv, d, page):
    """Pages of a tile, and tiles, whose scales are many powers of two apart, zeros and subnormal numbers among them."""
    new, lens = [40, 3, 1], [400, 650, 90]
    for dtype in TYPES:
        for seed, spread in ((1, 3), (2, 12), (3, 30)):
            pages = Pages(lens, hkv, d, page, 47 + seed)
            rng = np.random.default_rng(seed)
            pages.scales[1][:] = torch.from_numpy((2.0 ** rng.uniform(-spread, spread, tuple(pages.scales[1].shape))).astype(np.float32)).cuda() * 0.01
            pages.scales[1][pages.table[0, 1]] = 0.0
            pages.scales[1][pages.table[1, 2]] = 2.0 ** -130
            pages.scales[0][pages.table[0, 0]] = 0.0
            check(api, pages, queries(sum(new), hq, d, dtype, 3, 1.0 if spread < 30 else 0.3), lens, new)


@pytest.mark.parametrize("order", ["rising", "falling"])
def test_chunk_every_scale_counts(api, order):
    """Values of each page in a dimension of its own: what a page adds is seen beside pages that are larger by any factor up to 2^50."""
    page, d, n = 16, 64, 16 * 26
    pages = Pages([n], 1, d, page, 53)
    pages.codes[1][:] = 0
    for i in range(26):
        j = i if order == "rising" else 25 - i
        pages.codes[1][pages.table[0, i], 0, :, i] = 100
        pages.scales[1][pages.table[0, i]] = 2.0 ** (2 * j - 30)
    for new in (1, 20, 200):
        q = queries(new, 2, d, torch.bfloat16, 57, 0.5)
        got = check(api, pages, q, [n], [new])
        seen = (f64(got[:, :, :13]) > 0)
        assert seen.all()


@pytest.mark.parametrize("first,new,most", [(30, [70, 4], 0), (3, [8, 4], 8)])
def test_chunk_what_is_not_attended_to_has_no_influence(api, first, new, most):
    """Codes and scales of later tokens, of slots behind the end, of pages that are not reached; pages that read as NaN."""
    page, last = 32, new[0]
    lens = [160 - first + last, 75]  # token 160 is new token `first`
    for dtype in TYPES:
        pages = Pages(lens, 2, 64, page, 59)
        q = queries(sum(new), 4, 64, dtype, 61)
        run = lambda: api.pd_attn_chunk(q, *pages.tensors(), offsets(new), i32(lens), pages.block_table, most)  # noqa: E731
        clean = run()
        end = pages.table[0, lens[0] // page]
        pages.codes[0][end, :, lens[0] % page:] = 77
        pages.codes[1][end, :, lens[0] % page:] = -77
        assert torch.equal(run(), clean)
        for which in (0, 1):
            for bad in (float("nan"), float("inf")):
                held = pages.scales[which][pages.table[0, 5], 1].clone()
                pages.scales[which][pages.table[0, 5], 1] = bad  # tokens 160 .. 191
                got = run()
                pages.scales[which][pages.table[0, 5], 1] = held
                assert bool(torch.isnan(got[first:last, 2:].float()).all())
                assert torch.equal(got[:first], clean[:first]) and torch.equal(got[:, :2], clean[:, :2]) and torch.equal(got[last:], clean[last:])


def test_chunk_strides_and_untouched_rows(api):
    new, lens = [40, 2], [90, 33]
    pages = Pages(lens, 2, 64, 32, 67)
    wide = torch.randn(60, 11, 72, generator=torch.Generator("cuda").manual_seed(2), device="cuda").bfloat16()
    q = wide[:, 1:9, 8:]
    want = api.pd_attn_chunk(q[5:47].contiguous(), *pages.tensors(), offsets(new), i32(lens), pages.block_table)
    big = torch.full((60, 10, 80), 5.0, dtype=torch.bfloat16, device="cuda")
    api.pd_attn_chunk(q, *pages.tensors(), i32([5, 45, 47]), i32(lens), pages.block_table, out=big[:, 1:9, 8:72])
    assert torch.equal(big[5:47, 1:9, 8:72], want)
    big[5:47, 1:9, 8:72] = 5.0
    assert bool((big == 5.0).all())
    heads_first = q[5:47].transpose(0, 1).contiguous().transpose(0, 1)
    table = torch.full((2, pages.block_table.shape[1] + 5), -9, dtype=torch.int32, device="cuda")
    table[:, :pages.block_table.shape[1]] = pages.block_table
    assert torch.equal(api.pd_attn_chunk(heads_first, *pages.tensors(), offsets(new), i32(lens), table[:, :pages.block_table.shape[1]]), want)


@pytest.mark.parametrize("few", [False, True])
def test_chunk_bad_indices_are_reported(api, few):
    new, lens = ([50, 4], [100, 40]) if not few else ([6, 4], [100, 40])
    a, b = new[0], sum(new)
    pages = Pages(lens, 2, 64, 32, 71)
    q = queries(b, 4, 64, torch.float16, 73)
    call = lambda cu, n, table, most=8 if few else 0: api.pd_attn_chunk(q, *pages.tensors(), i32(cu), i32(n), table, most)  # noqa: E731
    for entry in (-1, pages.codes[0].shape[0], 2 ** 31 - 1):
        table = pages.block_table.clone()
        table[0, 2] = entry
        got = call([0, a, b], lens, table)
        assert api.pd_device_status(api.chunk_workspace()) == 8
        check(api, pages, q, lens, new, got=got, only=set(range(a, b)))
    bad = [([0, a, b], [a - 1, 40]), ([0, a, b], [pages.block_table.shape[1] * 32 + 1, 40]), ([0, a, b], [-5, 40]), ([0, b + 1, b], lens), ([-1, a, b], lens), ([0, a, b], [0, 40])]
    for cu, n in bad:
        call(cu, n, pages.block_table.clamp(min=0))
        assert api.pd_device_status(api.chunk_workspace()) == 8, (cu, n)
    call([0, a, b], lens, pages.block_table, a - 1)
    assert api.pd_device_status(api.chunk_workspace()) == 8
    assert api.pd_device_status(api.chunk_workspace()) == 0
    none = call([0, 0, 0], lens, pages.block_table)  # no new tokens: nothing to say
    assert none.shape == q.shape and api.pd_device_status(api.chunk_workspace()) == 0
    assert api.pd_attn_chunk(q[:0], *pages.tensors(), i32([0, 0, 0]), i32(lens), pages.block_table).shape == (0, 4, 64)


def test_chunk_agrees_with_single_tokens_and_prompts(api):
    """The three kinds of attention of the library on the same tokens: one at a time, a piece, a prompt of what the codes stand for."""
    hq, hkv, d, page, n = 8, 2, 128, 64, 333
    pages = Pages([n], hkv, d, page, 79)
    q = queries(n, hq, d, torch.float16, 83)
    piece = check(api, pages, q, [n], [n])
    one = api.pd_attn_cache(q[-1:], *pages.tensors(), i32([n]), pages.block_table)
    assert torch.equal(one, api.pd_attn_chunk(q[-1:], *pages.tensors(), offsets([1]), i32([n]), pages.block_table, 1))
    _, bound = definition(pages, f64(q), [n], [n], d ** -0.5, torch.float16, {n - 1})
    assert np.all(np.abs(f64(one[0]) - f64(piece[-1])) <= 2 * bound[-1])


def test_chunk_offsets_past_32_bits(api):
    """The last pages of a cache of more than 2^32 bytes."""
    hkv, d, page = 8, 128, 64
    n_pages = 2 ** 32 // (hkv * d * page) + 40
    codes = [torch.empty(n_pages, hkv, page, d, dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(n_pages, hkv, dtype=torch.float32, device="cuda") for _ in range(2)]
    k, v = (queries(150, hkv, d, torch.float16, i) for i in (1, 2))
    q = queries(150, 16, d, torch.float16, 3)
    small = [torch.zeros(3, hkv, page, d, dtype=torch.int8, device="cuda") for _ in range(2)] + [torch.zeros(3, hkv, device="cuda") for _ in range(2)]
    got = []
    for cache, table in ((codes + scales, i32([[n_pages - 1, n_pages - 30, n_pages - 7]])), (small, i32([[2, 0, 1]]))):
        turned = api.pd_kv_append_rope(q, k, v, *cache, offsets([150]), i32([150]), table, frequencies(64))
        got.append(api.pd_attn_chunk(turned, *cache, offsets([150]), i32([150]), table))
    assert torch.equal(*got)
    assert api.pd_device_status(api.attn_workspace()) == 0 and api.pd_device_status(api.chunk_workspace()) == 0
