"""Attention operators on the GPU at the ends of their ranges, against fp64 definitions.

Bound of pd_attn_cache, for each output, with w_j the weights and M the largest score of the row, L = sum_j e^(s_j - M):
  - rounding to the output's type: u_out |out| (u = 2^-11 for binary16, 2^-8 for bfloat16), and its smallest step;
  - P in binary16: 2^-11 sum_j w_j |v_j|; where P is subnormal 2^-25 of a unit, which is at most 64 page scales (the reference
    scale is at most 8 times a tile's largest, that at most 8 times the other one of the tile) and at most 1 / L of a weight,
    and never more than the weight itself: sum_j min(w_j, 2^-19 / L) |v_j|; where V's scales are 2^100 apart, what is far below does not count: 2^-90 of the largest |v_j|;
  - scores: a query is a multiple of 2^-21 of the power of two below its largest value, so that a score is off by
    d_j <= scale 2^-22 max|q| sum |k_j|; binary32 arithmetic adds 2^-20 (|s_j| + 1).  Weights are off by e^(2 max d) - 1 then."""
import numpy as np
import pytest
import torch

from oracle import pd_oracle_attn as orc

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


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def offsets(lens):
    return i32(np.concatenate([[0], np.cumsum(lens)]).tolist())


class Cache:
    """Pages of some sequences, one after another: codes int8 [pages, heads, page, d], scales [pages, heads]; numpy arrays."""

    def __init__(self, lens, hkv, d, page, seed):
        self.lens, self.page = lens, page
        rng = np.random.default_rng(seed)
        n = [-(-x // page) for x in lens]
        self.table, at = np.full((len(lens), max(n)), -1), 0
        for b, m in enumerate(n):
            self.table[b, :m] = np.arange(at, at + m)
            at += m
        self.k_codes, self.v_codes = (rng.integers(-127, 128, (at, hkv, page, d)).astype(np.int8) for _ in range(2))
        self.k_scale, self.v_scale = (np.exp(rng.normal(-4, 0.3, (at, hkv))).astype(np.float32) for _ in range(2))

    def device(self):
        return [torch.from_numpy(x).cuda() for x in (self.k_codes, self.v_codes, self.k_scale, self.v_scale)] + [i32(self.lens), i32(self.table.tolist())]

    def rows(self, b, g):
        """Codes of K and V and the scales of each token of sequence b, head g (fp64); V's scales below 2^-120 count as zero."""
        n, pages = self.lens[b], self.table[b, :-(-self.lens[b] // self.page)]
        flat = lambda x: x[pages, g].reshape(-1, x.shape[3])[:n].astype(np.float64)  # noqa: E731
        each = lambda x: np.repeat(x[pages, g].astype(np.float64), self.page)[:n]  # noqa: E731
        sv = each(self.v_scale)
        return flat(self.k_codes), flat(self.v_codes), each(self.k_scale), np.where(sv < 2.0 ** -120, 0.0, sv)

    def definition(self, q, scale, dtype):
        """Outputs and their bound for queries q (fp64) [B, Hq, d]."""
        out, bound = np.zeros_like(q), np.zeros_like(q)
        group = q.shape[1] // self.k_codes.shape[1]
        for b in range(len(self.lens)):
            for h in range(q.shape[1] if self.lens[b] else 0):
                if h % group == 0:
                    kc, vc, sk, sv = self.rows(b, h // group)
                    v, magnitude = vc * sv[:, None], np.abs(vc) * sv[:, None]
                    k_sum = np.abs(kc).sum(1) * sk
                s = (kc @ q[b, h]) * sk * scale
                e = np.exp(s - s.max())
                w = e / e.sum()
                off = (abs(scale) * 2.0 ** -22 * np.abs(q[b, h]).max() * k_sum + 2.0 ** -20 * (np.abs(s) + 1)).max()
                near = w @ magnitude
                out[b, h] = w @ v
                bound[b, h] = (UNIT[dtype] * np.abs(out[b, h]) + SMALLEST[dtype] + (2.0 ** -11 + np.expm1(2 * off)) * near +
                               np.minimum(w, 2.0 ** -19 / e.sum()) @ magnitude + 2.0 ** -90 * magnitude.max())
        return out, bound

    def without(self, q, scale, b, h):
        """Row (b, h) with each of its 32-token tiles left out: [tiles, d]."""
        kc, vc, sk, sv = self.rows(b, h * self.k_codes.shape[1] // q.shape[1])
        s = (kc @ q[b, h]) * sk * scale
        e, at = np.exp(s - s.max()), np.arange(0, len(s), 32)
        total, value = np.add.reduceat(e, at), np.add.reduceat((e * sv)[:, None] * vc, at)
        return (value.sum(0) - value) / (total.sum() - total)[:, None]


def check(got, want, bound):
    got = f64(got)
    assert np.all(np.isfinite(got))
    assert np.all(np.abs(got - want) <= bound), float((np.abs(got - want) / bound).max())


def attend(api, cache, q, scale):
    got = api.pd_attn_cache(q, *cache.device(), scale)
    assert api.pd_device_status(api.attn_workspace()) == 0
    return got


# ------------------------------------------------------------------ scales of V at the ends of their range
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 128), (12, 1, 64), (4, 4, 64)])
@pytest.mark.parametrize("page", [16, 64])
def test_cache_values_with_scales_of_any_size(api, hq, hkv, d, page):
    """Pages of V that are below 2^-120 (zeros), just above it, or far above or below the others, in every order."""
    n = 12 * page + 3
    scales = [[2.0 ** -126] * 13, [1e-38, 1.0] + [1e-38] * 11, [1.0] * 6 + [2.0 ** -119] * 7, [2.0 ** -119] * 6 + [1.0] * 7, [3e4] * 8 + [1e-36] * 5,
              [2.0 ** (16 * (6 - i)) for i in range(13)], [2.0 ** (16 * (i - 6)) for i in range(13)], [1.0, 0.0, 2.0 ** -100, 0.0] * 3 + [1.0]]
    cache = Cache([n] * len(scales), hkv, d, page, 5)
    for b, of_pages in enumerate(scales):
        cache.v_scale[cache.table[b]] = np.array(of_pages, dtype=np.float32)[:, None]
    q = torch.randn(len(scales), hq, d, generator=torch.Generator("cuda").manual_seed(hq), device="cuda").bfloat16()
    want, bound = cache.definition(f64(q), d ** -0.5, torch.bfloat16)
    check(attend(api, cache, q, d ** -0.5), want, bound)
    assert not want[0].any() and np.median(bound[1:5] / np.abs(want[1:5])) < 0.05


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 128), (12, 1, 64), (32, 2, 128)])
def test_cache_pages_of_a_tile_with_very_different_scales(api, hq, hkv, d, dtype):
    """Pages of 16 tokens, every other one with values far above the rest and with keys that hardly any head attends to: what the
    heads do attend to is not rounded by the neighbours' scale."""
    lens = [16 * 9 + 5, 16 * 40, 31]
    apart = {torch.float16: (2.0 ** 14, 2.0 ** -10), torch.bfloat16: (2.0 ** 30, 2.0 ** -30)}[dtype]
    for odd in (0, 1):
        cache = Cache(lens, hkv, d, 16, 37)
        large = (np.arange(len(cache.k_codes)) + odd) % 2 == 0
        cache.v_scale[large], cache.v_scale[~large] = np.float32(apart[0] / 127), np.float32(apart[1])
        cache.k_codes[large, :, :, 0], cache.k_codes[~large, :, :, 0] = -127, 0
        q = torch.randn(len(lens), hq, d, generator=torch.Generator("cuda").manual_seed(41), device="cuda").to(dtype)
        q[..., 0] = 800.0
        want, bound = cache.definition(f64(q), d ** -0.5, dtype)
        assert np.abs(want[1]).max() < 2.0 ** 8 * apart[1] and np.median(bound[1]) < 0.1 * np.sqrt(np.mean(want[1] ** 2))
        check(attend(api, cache, q, d ** -0.5), want, bound)


@pytest.mark.parametrize("lens", [[333], [7, 9000], [640] * 40], ids=["333", "7, 9000", "40 x 640"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 8, 128), (16, 1, 64)])
@pytest.mark.parametrize("exponent", [121, 100, -90])
def test_cache_values_at_the_ends_of_bfloat16(api, exponent, hq, hkv, d, lens):
    """Means of values up to 127 * 2^121, which is near bfloat16's largest, are finite, however the sequence is cut."""
    cache = Cache(lens, hkv, d, 64, 79)
    cache.v_scale[:] = 2.0 ** exponent
    q = torch.randn(len(lens), hq, d, generator=torch.Generator("cuda").manual_seed(83), device="cuda").bfloat16()
    want, bound = cache.definition(f64(q), 0.05, torch.bfloat16)
    check(attend(api, cache, q, 0.05), want, bound)


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 128), (12, 1, 64), (16, 2, 128)])
@pytest.mark.parametrize("first,then", [(2.0 ** 100, 2.0 ** -119), (2.0 ** 60, 2.0 ** -119), (1.0, 2.0 ** -119), (2.0 ** -119, 2.0 ** 100)])
@pytest.mark.parametrize("leads", [(30.0, 10.0, -30.0, 0.0), (30.0, 25.0, 28.0, 30.0), (150.0, 140.0, 150.0, 150.0)], ids=["some", "all", "far"])
def test_cache_weights_that_vanish_beside_scales_that_fall(api, leads, first, then, hq, hkv, d):
    """Some heads, or all of them, leave the first pages behind by up to e^300 when the scales of V change: every sequence is whole in a warp."""
    n_seqs, page = 1600, 32
    cache = Cache([4 * page] * n_seqs, hkv, d, page, 89)
    early = np.arange(4 * n_seqs) % 4 < 2
    cache.v_scale[early], cache.v_scale[~early], cache.k_scale[:] = np.float32(first), np.float32(then), 2.0 ** -6
    cache.k_codes[early, ..., 0], cache.k_codes[~early, ..., 0] = -64, 64
    q = 0.1 * torch.randn(n_seqs, hq, d, generator=torch.Generator("cuda").manual_seed(97), device="cuda")
    q[..., 0] = torch.tensor(leads, device="cuda").repeat(hq // 4)
    q = q.bfloat16()
    got = attend(api, cache, q, 1.0)
    assert bool(torch.isfinite(got).all())
    some = [0, 1, 77, n_seqs - 1]
    part = Cache([4 * page] * len(some), hkv, d, page, 0)
    for name in ("k_codes", "v_codes", "k_scale", "v_scale"):
        setattr(part, name, getattr(cache, name)[cache.table[some].reshape(-1)])
    want, bound = part.definition(f64(q[some]), 1.0, torch.bfloat16)
    check(got[some], want, bound)


def test_appended_values_that_are_tiny(api):
    """What pd_kv_append writes for values near 1e-38 reads as zeros, before, after and without ordinary pages."""
    d, page, n = 64, 32, 96
    gen = torch.Generator("cuda").manual_seed(9)
    k, q = torch.randn(n, 1, d, generator=gen, device="cuda").bfloat16(), torch.randn(1, 2, d, generator=gen, device="cuda").bfloat16()
    for tiny in ([0, 1, 2], [0], [1], [2]):
        v = torch.ones(n, 1, d, dtype=torch.bfloat16, device="cuda")
        for i in tiny:
            v[i * page:(i + 1) * page] = 1e-38
        tensors = [torch.zeros(3, 1, page, d, dtype=torch.int8, device="cuda") for _ in range(2)] + [torch.zeros(3, 1, device="cuda") for _ in range(2)]
        api.pd_kv_append(k, v, *tensors, offsets([n]), i32([n]), i32([[0, 1, 2]]))
        got = f64(api.pd_attn_cache(q, *tensors, i32([n]), i32([[0, 1, 2]])))
        cache = Cache([n], 1, d, page, 0)
        cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale = (t.cpu().numpy() for t in tensors)
        want, bound = cache.definition(f64(q), d ** -0.5, torch.bfloat16)
        assert np.all(np.abs(got - want) <= bound) and (len(tiny) < 3 or not got.any())


# ------------------------------------------------------------------ queries of any size
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 128), (12, 1, 64)])
def test_cache_queries_at_the_ends_of_bfloat16(api, hq, hkv, d):
    """A query times a power of two with the scale divided by it gives the same bits, from the smallest normal exponent to the largest."""
    cache = Cache([70, 333, 1], hkv, d, 32, 11)
    gen = torch.Generator("cuda").manual_seed(13)
    q = torch.rand(3, hq, d, generator=gen, device="cuda").bfloat16() * 0.984375 + 1.0  # magnitudes in [1, 2)
    assert float(q.min()) >= 1 and float(q.max()) < 2
    q *= torch.randint(0, 2, q.shape, generator=gen, device="cuda").bfloat16() * 2 - 1
    for scale, powers in ((2.0 ** -3, (-101, -113, -120, -126)), (16.0, (99, 101, 102, 103, 110, 125, 127))):
        if scale > 1:
            cache.k_scale *= np.float32(2.0 ** -7)
        clean = attend(api, cache, q, scale)
        want, bound = cache.definition(f64(q), scale, torch.bfloat16)
        check(clean, want, bound)
        for e in powers:
            big = (q.double() * 2.0 ** e).bfloat16()
            assert torch.equal(big.double(), q.double() * 2.0 ** e)
            assert torch.equal(attend(api, cache, big, scale * 2.0 ** -e), clean), e
    for bad in (float("inf"), -float("inf"), float("nan")):
        big = q.clone()
        big[1, 0, 7] = bad
        got = attend(api, cache, big, 2.0 ** -3)
        assert bool(torch.isnan(got[1, 0]).all()) and bool(torch.isfinite(got[1, 1:]).all()) and bool(torch.isfinite(got[0]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("factor", [2.0 ** 6, 2.0 ** 9])
def test_cache_query_with_one_large_channel(api, dtype, factor):
    """Most of a head's query is far below its largest value; the keys hardly use that channel, so that the rest decides."""
    cache = Cache([500, 90], 2, 128, 64, 17)
    cache.k_codes[..., 5] = np.sign(cache.k_codes[..., 5])
    q = torch.randn(2, 4, 128, generator=torch.Generator("cuda").manual_seed(19), device="cuda").to(dtype)
    q[..., 5] = factor
    want, bound = cache.definition(f64(q), 0.3, dtype)
    assert np.median(bound) < 0.04 * np.sqrt(np.mean(want ** 2))
    check(attend(api, cache, q, 0.3), want, bound)


# ------------------------------------------------------------------ offsets and lengths out of range
def append_ones(api, cu, lens, n_tokens, page):
    """The status after appending ones to an empty cache."""
    d, width = 64, -(-max(lens) // page)
    x = torch.ones(n_tokens, 1, d, dtype=torch.float16, device="cuda")
    tensors = [torch.zeros(len(lens) * width, 1, page, d, dtype=torch.int8, device="cuda") for _ in range(2)] + [torch.zeros(len(lens) * width, 1, device="cuda") for _ in range(2)]
    api.pd_kv_append(x, x, *tensors, i32(cu), i32(lens), torch.arange(len(lens) * width, dtype=torch.int32, device="cuda").view(-1, width))
    return api.pd_device_status(api.attn_workspace())


@pytest.mark.parametrize("page", [16, 128])
def test_append_reports_offsets_that_decrease(api, page):
    for cu, lens in (([0, 1000, 0, 50], [1000, 10, 50]), ([0, 40, 30, 1000], [40, 10, 970]), ([0, 500, 1000, 999, 1000], [500, 500, 0, 1])):
        assert append_ones(api, cu, lens, 1000, page) == 8, cu


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("new", [1, 5])
def test_append_reports_one_bad_pair_among_many(api, new, page):
    """Single tokens (a warp per sequence) and pieces (a block per page): one sequence reaches to the end, the next one down again."""
    n, cu = 200, [new * i for i in range(201)]
    assert append_ones(api, cu, [new] * n, cu[-1], page) == 0
    for at in (0, 1, 30, 31, 32, 100, 198):
        bad = list(cu)
        bad[at + 1] = cu[-1] - (at < 198) if at < 198 else cu[at] - 1
        lens = [max(b - a, new) for a, b in zip(bad, bad[1:])]
        assert min(b - a for a, b in zip(bad, bad[1:])) < 0
        assert append_ones(api, bad, lens, cu[-1], page) == 8, at


@pytest.mark.parametrize("hkv,d", [(2, 64), (4, 128)])
def test_prompt_takes_no_sequence_behind_offsets_that_decrease(api, hkv, d):
    """Sequences that have tokens in common could be any amount of work: only those before the offsets go down are computed."""
    gen = torch.Generator("cuda").manual_seed(23)
    q, k, v = (torch.randn(400, h, d, generator=gen, device="cuda").half() for h in (4, hkv, hkv))
    alone = api.pd_attn_prompt(q[:100].contiguous(), k[:100].contiguous(), v[:100].contiguous(), offsets([100]))
    assert api.pd_device_status(api.attn_workspace()) == 0
    for cu in ([0, 100, 50, 150], [0, 100] + [20, 400] * 40, [0] * 40 + [100, 90] + list(range(90, 400, 10))):
        out = torch.full((400, 4, d), 7.0, dtype=torch.float16, device="cuda")
        api.pd_attn_prompt(q, k, v, i32(cu), out=out)
        assert api.pd_device_status(api.attn_workspace()) == 8
        assert torch.equal(out[:100], alone) and bool((out[100:] == 7).all()), cu
    # out of range without going down: the others are served
    for cu, keep in (([-5, 0, 100], (0, 100)), ([0, 100, 401, 402], (0, 100))):
        out = torch.full((400, 4, d), 7.0, dtype=torch.float16, device="cuda")
        api.pd_attn_prompt(q, k, v, i32(cu), out=out)
        assert api.pd_device_status(api.attn_workspace()) == 8
        assert torch.equal(out[:100], alone) and bool((out[100:] == 7).all()), cu


# ------------------------------------------------------------------ infinities and NaN among the keys
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("at", [64, 70, 20])
def test_a_key_that_is_not_finite_reads_as_nan(api, at, bad, dtype):
    """Alone in its page, among others, appended in one call or by itself, whatever the sign of the query: NaN, and codes of zero."""
    d, page, n = 64, 32, at + 1 if at > 32 else 65
    gen = torch.Generator("cuda").manual_seed(29)
    k, v = (torch.randn(n, 2, d, generator=gen, device="cuda").to(dtype) for _ in range(2))
    k[at, 1, 9] = bad
    q = torch.randn(1, 4, d, generator=gen, device="cuda").to(dtype)
    table = i32([[2, 0, 1]])
    for steps in ([n], [at, n - at], [at] + [1] * (n - at)):
        tensors = [torch.full((3, 2, page, d), 55, dtype=torch.int8, device="cuda") for _ in range(2)] + [torch.zeros(3, 2, device="cuda") for _ in range(2)]
        held = 0
        for m in steps:
            values = torch.empty(m, 2, d, dtype=dtype, device="cuda")
            api.pd_kv_append(k[held:held + m].contiguous(), v[held:held + m].contiguous(), *tensors, offsets([m]), i32([held + m]), table, values)
            held += m
        p = [2, 0, 1][at // page]
        assert not tensors[0][p, 1, :min(page, n - at // page * page)].any()
        scale = float(tensors[2][p, 1])
        assert scale != scale if bad != bad else scale == float("inf")
        if at // page == (n - 1) // page:  # the values of the last call's tokens in that page
            assert bool(torch.isnan(values[max(at // page * page - (n - m), 0):, 1]).all())
        for sign in (1, -1):
            query = q.clone()
            query[:, 2:, 9] = sign * 2.0
            got = api.pd_attn_cache(query, *tensors, i32([n]), table)
            assert bool(torch.isnan(got[:, 2:]).all()) and bool(torch.isfinite(got[:, :2]).all())
    assert api.pd_device_status(api.attn_workspace()) == 0


# ------------------------------------------------------------------ scales of scores
@pytest.mark.parametrize("hkv,d", [(2, 64), (4, 128)])
def test_prompt_with_a_scale_of_zero_and_large_scores(api, hkv, d):
    """Scores up to 1e37 times zero are zero: means of the values so far.  exp2(2^-21) is off by 2^-21 and is covered by 2^-20 of the mean magnitude."""
    lens = [150, 290]
    gen = torch.Generator("cuda").manual_seed(31)
    q, k, v = (torch.randn(sum(lens), h, d, generator=gen, device="cuda").bfloat16() for h in (4, hkv, hkv))
    got = f64(api.pd_attn_prompt(q * 2.0 ** 58, k * 2.0 ** 58, v, offsets(lens), 0.0))
    zero, vd = np.zeros_like(f64(q)), f64(v)
    want = orc.attn_prompt(zero, np.zeros_like(vd), vd, lens, 0.0)
    near = orc.attn_prompt(zero, np.zeros_like(vd), np.abs(vd), lens, 0.0)
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -20) * near)


@pytest.mark.parametrize("dtype,sizes", [(torch.float16, (300.0, 3000.0, 15000.0)), (torch.bfloat16, (300.0, 1e5, 1e9, 1e14))], ids=["fp16", "bf16"])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (3, 3, 128)])
def test_prompt_with_scores_of_any_size(api, hq, hkv, d, dtype, sizes):
    """Finite scores give finite outputs, however large: nearly always all of the weight is one token's.  A score is off by at most
    2^-18 sum_d |q_d k_d| of the sums and products in binary32, and weights by e^(twice that)."""
    lens = [300, 77]
    gen = torch.Generator("cuda").manual_seed(67)
    q, k, v = (torch.randn(sum(lens), h, d, generator=gen, device="cuda") for h in (hq, hkv, hkv))
    for size in sizes:
        most = 6e4 if dtype == torch.float16 else 3e38  # so that they are finite
        qs, ks, vs = (q * size).clamp(-most, most).to(dtype), (k * size).clamp(-most, most).to(dtype), v.to(dtype)
        for scale in (d ** -0.5, -0.3):
            got = f64(api.pd_attn_prompt(qs, ks, vs, offsets(lens), scale))
            assert np.all(np.isfinite(got))
            want, near, sure = np.zeros_like(got), np.zeros_like(got), np.zeros(got.shape[:2], bool)
            qd, kd, vd, at = f64(qs), np.repeat(f64(ks), hq // hkv, axis=1), np.repeat(f64(vs), hq // hkv, axis=1), 0
            for n in lens:
                for h in range(hq):
                    s = qd[at:at + n, h] @ kd[at:at + n, h].T * scale
                    off = np.abs(qd[at:at + n, h]) @ np.abs(kd[at:at + n, h]).T * abs(scale) * 2.0 ** -18
                    s = np.where(np.tri(n, dtype=bool), s, -np.inf)
                    w = np.exp(s - s.max(axis=1, keepdims=True))
                    w /= w.sum(axis=1, keepdims=True)
                    want[at:at + n, h], near[at:at + n, h] = w @ vd[at:at + n, h], w @ np.abs(vd[at:at + n, h])
                    # rows where the largest score is larger than the others by more than what both may be off, and 30
                    low = np.where(np.tri(n, dtype=bool), s + off, -np.inf)
                    best = s.argmax(axis=1)
                    low[np.arange(n), best] = -np.inf
                    sure[at:at + n, h] = s.max(axis=1) - off[np.arange(n), best] > low.max(axis=1) + 30
                at += n
            assert sure.mean() > 0.9
            assert np.all(np.abs(got - want)[sure] <= (UNIT[dtype] * np.abs(want) + (UNIT[dtype] + 2.0 ** -14) * near)[sure])


def test_cache_scores_whose_spacing_passes_the_lead(api):
    """Scores near 2^27 (base 2), 16 apart in binary32: a tile that leads by one step moves the reference maximum, whatever that rounds to.
    Every sequence is whole in one warp, which goes through its two tiles in turn."""
    d, n_seqs, hkv = 64, 96, 32
    cache = Cache([64] * n_seqs, hkv, d, 32, 71)
    cache.k_codes[:], cache.k_scale[:], cache.v_scale[:] = 0, 1.0, 1.0
    cache.k_codes[..., 0] = 127
    for b in range(n_seqs):
        cache.k_codes[cache.table[b, 0], ..., 1], cache.k_codes[cache.table[b, 1], ..., 1] = b, b + 1
    cache.v_codes[0::2], cache.v_codes[1::2] = 1, -1
    q = torch.zeros(n_seqs, hkv, d, dtype=torch.bfloat16, device="cuda")
    q[..., 0], q[..., 1] = 750000.0, 11.0
    got = f64(attend(api, cache, q, 1.0))
    assert np.all(np.abs(got) <= 1)


def test_prompt_scores_whose_spacing_passes_the_lead(api):
    """The same of prompts in binary16: each tile of 128 keys leads the one before by 8 in a score near 2^26.5."""
    n, d = 1280, 64
    for start in range(0, 64, 8):
        q, k, v = (torch.zeros(n, 2, d, dtype=torch.float16, device="cuda") for _ in range(3))
        q[..., 0], k[..., 0], q[..., 1] = 30000.0, 3130.0, 1.0
        k[..., 1] = (start + 8 * (torch.arange(n, device="cuda") // 128))[:, None].half()
        v[:] = torch.where(torch.arange(n, device="cuda") // 128 % 2 == 0, 1.0, -1.0)[:, None, None].half()
        got = f64(api.pd_attn_prompt(q, k, v, offsets([n]), 1.0))
        assert np.all(np.abs(got) <= 1)


@pytest.mark.parametrize("hkv,d", [(2, 64), (4, 128)])
@pytest.mark.parametrize("exponent", [127, 100, -90])
def test_prompt_values_at_the_ends_of_bfloat16(api, hkv, d, exponent):
    """Means of finite values are finite, up to the largest that bfloat16 has, and small ones keep their precision."""
    lens = [1500, 90]
    gen = torch.Generator("cuda").manual_seed(73)
    q, k, v = (torch.randn(sum(lens), h, d, generator=gen, device="cuda") for h in (4, hkv, hkv))
    q, k, v = q.bfloat16(), k.bfloat16(), ((v * 0.3).clamp(-1, 1) * 1.9921875 * 2.0 ** exponent).bfloat16()
    assert bool(torch.isfinite(v).all())
    got, vd = f64(api.pd_attn_prompt(q, k, v, offsets(lens))), f64(v)
    rows = list(range(0, 1500, 50)) + [1499, 1500, 1501, 1589]
    for i in rows:
        first = 0 if i < 1500 else 1500
        for h in range(4):
            s = f64(k[first:i + 1, h * hkv // 4]) @ f64(q[i, h]) * d ** -0.5
            w = np.exp(s - s.max())
            w /= w.sum()
            x = vd[first:i + 1, h * hkv // 4]
            assert np.all(np.abs(got[i, h] - w @ x) <= 2.0 ** -8 * np.abs(w @ x) + (2.0 ** -8 + 2.0 ** -14) * (w @ np.abs(x)))


@pytest.mark.parametrize("hkv,d", [(2, 64), (4, 128)])
@pytest.mark.parametrize("gap", [16.6, 20.6, 23.42, 25.2])
def test_prompt_many_small_weights_beside_a_large_one(api, hkv, d, gap):
    """A prompt in binary16 whose first token holds nearly all of the weight, the others the rest, which is what the outputs are made
    of.  Each of them loses at most 2^-32 of the first one's weight."""
    n = 6000
    q, k = torch.zeros(n, 4, d, dtype=torch.float16, device="cuda"), torch.zeros(n, hkv, d, dtype=torch.float16, device="cuda")
    v = torch.rand(n, hkv, d, generator=torch.Generator("cuda").manual_seed(47), device="cuda").half() + 1000
    q[..., 3], k[0, :, 3], v[0] = 1.0, 1.0, 0.0
    scale = float(np.float32(gap * np.log(2)))
    got = f64(api.pd_attn_prompt(q, k, v, offsets([n]), scale))
    vd = np.repeat(f64(v), 4 // hkv, axis=1)
    w = np.exp(-scale) / (1 + np.exp(-scale) * np.arange(n))[:, None, None]  # of each token but the first
    want = w * np.cumsum(vd, axis=0)
    assert np.all(np.abs(got - want)[1:] <= ((2 * 2.0 ** -11 + 2.0 ** -14) * want + 2.0 ** -24 + 2.0 ** -32 * np.arange(n)[:, None, None] * 1001)[1:])
    assert 2.0 ** -32 < 0.01 * np.exp(-scale)


# ------------------------------------------------------------------ long sequences, cut into parts
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens", [[333], [7, 9000], [20011], [640] * 40], ids=["333", "7, 9000", "20011", "40 x 640"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 8, 128), (16, 2, 64), (32, 2, 128), (40, 1, 128), (1, 1, 64)])
def test_cache_every_tile_counts(api, hq, hkv, d, lens, dtype):
    """The work of a sequence is cut into parts that are joined.  A tile's values are in one dimension of the output, which it shares
    with few others, so that the bound would catch any tile that is lost or counted twice: checked of the definition here."""
    cache = Cache(lens, hkv, d, 64, 53)
    tile = np.arange(cache.table.shape[1] * 64).reshape(-1, 64) // 32
    for b in range(len(lens)):
        n = -(-lens[b] // 64)
        one = (np.arange(d) == tile[:n, :, None] % d)[:, None]
        cache.v_codes[cache.table[b, :n]] = one * (64 + np.abs(cache.v_codes[cache.table[b, :n]].astype(np.int64)) // 2)
    q = torch.randn(len(lens), hq, d, generator=torch.Generator("cuda").manual_seed(59), device="cuda").to(dtype)
    want, bound = cache.definition(f64(q), 0.02, dtype)
    assert np.median(bound[want > 0] / want[want > 0]) < 2.5 * (UNIT[dtype] + 2.0 ** -11)
    for b in {0, len(lens) - 1}:
        for h in {0, hq - 1}:
            assert (want[b, h] > 2 * bound[b, h]).any()
            if lens[b] > 32:
                assert np.all((np.abs(cache.without(f64(q), 0.02, b, h) - want[b, h]) > 2 * bound[b, h]).any(axis=1))
    got = attend(api, cache, q, 0.02)
    check(got, want, bound)
    assert torch.equal(got, attend(api, cache, q, 0.02))


# ------------------------------------------------------------------ forms of calls that a server makes
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [[1] * 63 + [190], [190] + [1] * 63, [1, 0, 0, 77, 1, 1, 0, 1] * 5, [0] * 30 + [100] + [0] * 9], ids=["end", "start", "some", "one"])
def test_append_of_single_tokens_with_longer_pieces(api, new, dtype):
    """Decode tokens and a piece of a prompt in one call: the same bits as each sequence by itself."""
    hkv, d, page = 2, 128, 32
    held = [(37 * b) % 100 for b in range(len(new))]
    total = [a + b for a, b in zip(held, new)]
    width = max(total) // page + 1
    gen = torch.Generator("cuda").manual_seed(61)
    kv = torch.randn(sum(new), 2 * hkv, d, generator=gen, device="cuda").to(dtype)
    wide = torch.arange(len(new) * (width + 3), dtype=torch.int32, device="cuda").view(len(new), width + 3).flip(0)
    table = wide[:, :width]  # rows further apart than they are wide
    codes = torch.randint(-127, 128, (wide.numel(), hkv, page, d), generator=gen, device="cuda", dtype=torch.int8)
    scale = torch.rand(wide.numel(), hkv, generator=gen, device="cuda") * 0.03

    def fresh():
        return [codes.clone(), codes.flip(0).contiguous(), scale.clone(), scale.flip(0).contiguous()]
    together, single = fresh(), fresh()
    values = [torch.empty(sum(new), hkv, d, dtype=dtype, device="cuda") for _ in range(2)]
    api.pd_kv_append(kv[:, :hkv], kv[:, hkv:], *together, offsets(new), i32(total), table, *values)
    at = 0
    for b, m in enumerate(new):
        if m:
            x = kv[at:at + m]
            out = [torch.empty(m, hkv, d, dtype=dtype, device="cuda") for _ in range(2)]
            api.pd_kv_append(x[:, :hkv], x[:, hkv:], *single, offsets([m]), i32(total[b:b + 1]), table[b:b + 1].contiguous(), *out)
            assert torch.equal(values[0][at:at + m], out[0]) and torch.equal(values[1][at:at + m], out[1])
            at += m
    assert api.pd_device_status(api.attn_workspace()) == 0
    assert all(torch.equal(x, y) for x, y in zip(together, single))
    q = torch.randn(len(new), 4, d, generator=gen, device="cuda").to(dtype)
    assert torch.equal(api.pd_attn_cache(q, *together, i32(total), table), api.pd_attn_cache(q, *together, i32(total), table.contiguous()))
