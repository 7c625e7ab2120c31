"""Attention operators on the GPU (pd_attn_prompt, pd_kv_append, pd_attn_cache) against fp64 definitions.

Tolerances, for each output: the result is rounded once to its type (relative u = 2^-11 for binary16, 2^-8 for bfloat16); the
weights are rounded to 16 bits before their product with v (relative u of that type each: the error of the sum is at most
u * sum_j w_j |v_j|); scores, exponentials and sums are binary32 (scores up to about 30 from products summed over 128 terms:
absolute error below 2^-15, so a relative error of the weights below 2^-14); weights below 2^-14 of the largest in binary16 lose
at most 2^-25 each.  Codes: three binary32 roundings of numbers up to 127 (2.3e-5) beside the half step."""
import numpy as np
import pytest
import torch

from oracle import pd_oracle_attn as orc

pytestmark = pytest.mark.gpu
UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
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


def close(got, want, weight_abs, u_out, u_p, extra=0.0):
    """|got - want| within the derived bound at every output; weight_abs: sum_j w_j |v_j|."""
    bound = u_out * np.abs(want) + (u_p + 2.0 ** -14) * weight_abs + extra + 1e-30
    off = np.abs(got - want) / bound
    assert np.all(np.isfinite(got)) and off.max() <= 1.0, float(off.max())


# ------------------------------------------------------------------ prompts
def prompt_inputs(lens, hq, hkv, d, dtype, seed, sd=1.0):
    gen = torch.Generator("cuda").manual_seed(seed)
    qkv = torch.randn(max(sum(lens), 1), hq + 2 * hkv, d, generator=gen, device="cuda").to(dtype)[:sum(lens)]
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    q.mul_(sd)
    return q, k, v


def check_prompt(got, q, k, v, lens, scale, dtype):
    want = orc.attn_prompt(f64(q), f64(k), f64(v), lens, scale)
    near = orc.attn_prompt(f64(q), f64(k), np.abs(f64(v)), lens, scale)
    close(f64(got), want, near, UNIT[dtype], UNIT[dtype], 2.0 ** -25 * max(lens) * np.abs(f64(v)).max() if dtype == torch.float16 else 0.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hkv,d", [(4, 4, 128), (8, 2, 64), (6, 2, 128), (5, 1, 64)])
@pytest.mark.parametrize("lens", [[1], [17], [64, 0, 65, 1, 127], [128, 129, 2], [300]], ids=str)
def test_prompt_matches_the_definition(api, lens, hq, hkv, d, dtype):
    q, k, v = prompt_inputs(lens, hq, hkv, d, dtype, 7 + sum(lens))
    got = api.pd_attn_prompt(q, k, v, offsets(lens))
    assert api.pd_device_status(api.attn_workspace()) == 0
    check_prompt(got, q, k, v, lens, d ** -0.5, dtype)
    assert torch.equal(got, api.pd_attn_prompt(q, k, v, offsets(lens)))  # the same bits again


@pytest.mark.parametrize("dtype", TYPES)
def test_prompt_large_scores_and_given_scale(api, dtype):
    lens = [200, 77]
    q, k, v = prompt_inputs(lens, 4, 2, 64, dtype, 3, sd=3.0)  # scores of 3 * 8 / 8 * N(0, 1) * 1.2: up to about 15
    check_prompt(api.pd_attn_prompt(q, k, v, offsets(lens), 0.15), q, k, v, lens, 0.15, dtype)
    check_prompt(api.pd_attn_prompt(q, k, v, offsets(lens), -0.15), q, k, v, lens, -0.15, dtype)
    check_prompt(api.pd_attn_prompt(q, k, v, offsets(lens), 0.0), q, k, v, lens, 0.0, dtype)  # means of the tokens so far


def test_prompt_rising_and_falling_scores(api):
    """Keys that make the running maximum grow at every tile, or never: both ways of the rescaling."""
    n, d = 513, 128
    for sign in (1.0, -1.0):
        q = torch.ones(n, 2, d, dtype=torch.float16, device="cuda")
        k = (sign * torch.arange(n, device="cuda")[:, None, None] / 8.0).expand(n, 2, d).to(torch.float16).contiguous()
        v = torch.randn(n, 2, d, generator=torch.Generator("cuda").manual_seed(5), device="cuda").half()
        got = api.pd_attn_prompt(q, k, v, offsets([n]), 0.01)  # scores up to 82: fp32 rounding of the score is below 2^-14 of a weight
        check_prompt(got, q, k, v, [n], 0.01, torch.float16)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("hkv,d", [(2, 128), (4, 128), (2, 64), (4, 64)])
def test_prompt_what_is_not_attended_to_has_no_influence(api, hkv, d, dtype, bad):
    lens = [70, 130, 33]
    q, k, v = prompt_inputs(lens, 4, hkv, d, dtype, 11)
    clean = api.pd_attn_prompt(q, k, v, offsets(lens))
    k2, v2 = k.clone(), v.clone()
    k2[65:70], v2[65:70] = bad, bad   # the last tokens of the first sequence
    v2[70 + 100, 1, 5] = bad          # one value in the middle of the second
    got = api.pd_attn_prompt(q, k2, v2, offsets(lens))
    keep = torch.ones_like(got, dtype=torch.bool)
    keep[65:70] = False
    heads = slice(4 // hkv, 8 // hkv)  # those that read key/value head 1
    keep[170:200, heads, 5] = False
    assert torch.equal(got[keep], clean[keep])
    hit = got[170:200, heads, 5].float()
    assert bool(torch.isnan(hit).all() if bad != bad else (hit == bad).all())
    assert bool(torch.isnan(got[65:70].float()).any())


def test_prompt_strides_and_untouched_rows(api):
    lens = [40, 90]
    q, k, v = prompt_inputs(lens, 8, 2, 64, torch.bfloat16, 13)
    want = api.pd_attn_prompt(q.contiguous(), k.contiguous(), v.contiguous(), offsets(lens))
    assert torch.equal(api.pd_attn_prompt(q, k, v, offsets(lens)), want)
    # heads before tokens, as after a transpose; the result into a wider tensor with more rows than the sequences claim
    kt, vt = k.transpose(0, 1).contiguous().transpose(0, 1), v.transpose(0, 1).contiguous().transpose(0, 1)
    wide = torch.full((130, 11, 80), 7.0, dtype=torch.bfloat16, device="cuda")
    out = wide[:, 2:10, 8:72]
    api.pd_attn_prompt(q, kt, vt, offsets(lens), out=out)
    assert torch.equal(out, want)
    wide[:, 2:10, 8:72] = 7.0
    assert bool((wide == 7.0).all())
    out = torch.full((130, 8, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    api.pd_attn_prompt(q, k, v, i32([3, 43, 43, 120]), out=out)  # offsets that start late and end early
    assert bool((out[:3] == 7.0).all() and (out[120:] == 7.0).all())
    want = api.pd_attn_prompt(q[3:43].contiguous(), k[3:43].contiguous(), v[3:43].contiguous(), offsets([40]))
    assert torch.equal(out[3:43], want)


def test_prompt_bad_offsets_are_reported(api):
    q, k, v = prompt_inputs([50], 2, 2, 64, torch.float16, 17)
    for cu in ([0, 30, 20, 50], [0, 51], [-1, 50]):
        api.pd_attn_prompt(q, k, v, i32(cu))
        assert api.pd_device_status(api.attn_workspace()) == 8
    assert api.pd_device_status(api.attn_workspace()) == 0
    assert api.pd_attn_prompt(q[:0], k[:0], v[:0], i32([0, 0])).shape == (0, 2, 64)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hkv,d", [(16, 4, 128), (12, 12, 128), (18, 6, 64)])
def test_prompt_long_sequences_on_samples(api, hq, hkv, d, dtype):
    """Thousands of tokens, many heads, next to short sequences: sampled queries against 64-bit sums."""
    lens = [2500, 3, 1111, 640]
    q, k, v = prompt_inputs(lens, hq, hkv, d, dtype, 19)
    got = api.pd_attn_prompt(q, k, v, offsets(lens))
    rng = np.random.default_rng(3)
    kd, vd, at = k.double(), v.double(), 0
    for n in lens:
        for i in sorted({0, n - 1, *rng.integers(0, n, 24).tolist()}):
            s = torch.einsum("hd,jhd->hj", q[at + i].double(), kd[at:at + i + 1].repeat_interleave(hq // hkv, dim=1)) * d ** -0.5
            w, vs = torch.softmax(s, dim=1), vd[at:at + i + 1].repeat_interleave(hq // hkv, dim=1)
            close(f64(got[at + i]), f64(torch.einsum("hj,jhd->hd", w, vs)), f64(torch.einsum("hj,jhd->hd", w, vs.abs())), UNIT[dtype], UNIT[dtype],
                  2.0 ** -25 * n * 5 if dtype == torch.float16 else 0.0)
        at += n


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (3, 3, 128)])
def test_prompt_many_sequences(api, hq, hkv, d):
    """More sequences than the lanes of a warp know at a time, some of them empty, some longer than a tile."""
    rng = np.random.default_rng(127)
    lens = [int(n) for n in rng.choice([0, 1, 2, 7, 31, 130], 75)]
    q, k, v = prompt_inputs(lens, hq, hkv, d, torch.float16, 131)
    got = api.pd_attn_prompt(q, k, v, offsets(lens))
    assert api.pd_device_status(api.attn_workspace()) == 0
    check_prompt(got, q, k, v, lens, d ** -0.5, torch.float16)


def test_prompt_again_and_again_gives_the_same_bits(api):
    """The blocks take their work in the order in which they come to it: the results do not depend on it."""
    lens = [700, 1300, 40, 511]
    q, k, v = prompt_inputs(lens, 16, 4, 128, torch.bfloat16, 137)
    first = api.pd_attn_prompt(q, k, v, offsets(lens))
    for _ in range(20):
        assert torch.equal(first, api.pd_attn_prompt(q, k, v, offsets(lens)))


# ------------------------------------------------------------------ the cache
class Pages:
    """A cache with its pages in random order; unused pages and table entries hold what must not be looked at."""

    def __init__(self, lens, hkv, d, page, seed, extra=3):
        self.rng = np.random.default_rng(seed)
        self.page, self.hkv, self.d = page, hkv, d
        n = [-(-x // page) for x in lens]
        self.n_pages = sum(n) + extra
        order = self.rng.permutation(self.n_pages)
        self.width = max(max(n), 1) + 2
        self.table = np.full((len(lens), self.width), -7, dtype=np.int64)
        at = 0
        for b, m in enumerate(n):
            self.table[b, :m] = order[at:at + m]
            at += m
        self.unused = order[at:]
        shape = (self.n_pages, hkv, page, d)
        self.k_codes = torch.from_numpy(self.rng.integers(-128, 128, shape).astype(np.int8)).cuda()
        self.v_codes = torch.from_numpy(self.rng.integers(-128, 128, shape).astype(np.int8)).cuda()
        self.k_scale = torch.from_numpy(np.exp(self.rng.normal(-4, 0.5, shape[:2])).astype(np.float32)).cuda()
        self.v_scale = torch.from_numpy(np.exp(self.rng.normal(-4, 1.5, shape[:2])).astype(np.float32)).cuda()
        bad = torch.from_numpy(self.unused).cuda()
        self.k_scale[bad], self.v_scale[bad] = float("nan"), float("inf")
        self.block_table = torch.from_numpy(self.table.astype(np.int32)).cuda()

    def tensors(self):
        return self.k_codes, self.v_codes, self.k_scale, self.v_scale

    def host(self):
        return [t.cpu().numpy() for t in self.tensors()]


def check_cache(got, q, pages, lens, scale, dtype):
    kc, vc, ks, vs = pages.host()
    want = orc.attn_cache(f64(q), kc, vc, ks, vs, lens, pages.table, scale)
    near = orc.attn_cache(f64(q), kc, np.abs(vc.astype(np.int64)), ks, vs, lens, pages.table, scale)
    used = vs[np.isfinite(vs)]
    extra = 2.0 ** -25 * 8 * max(lens) * 128 * (used.max() if used.size else 0)
    close(f64(got), want, near, UNIT[dtype], UNIT[torch.float16], extra)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hkv,d,page", [(4, 4, 128, 64), (8, 1, 128, 16), (6, 2, 64, 32), (12, 1, 128, 128), (16, 1, 64, 16), (40, 2, 128, 32)])
def test_cache_attention_matches_the_definition(api, hq, hkv, d, page, dtype):
    lens = [0, 1, page - 1, page, page + 1, 31, 33, 250, 0, 611]
    pages = Pages(lens, hkv, d, page, 23 + hq)
    q = torch.randn(len(lens), hq, d, generator=torch.Generator("cuda").manual_seed(hq), device="cuda").to(dtype)
    got = api.pd_attn_cache(q, *pages.tensors(), i32(lens), pages.block_table)
    assert api.pd_device_status(api.attn_workspace()) == 0
    check_cache(got, q, pages, lens, d ** -0.5, dtype)
    assert not got[0].any() and not got[8].any()
    for _ in range(3):
        assert torch.equal(got, api.pd_attn_cache(q, *pages.tensors(), i32(lens), pages.block_table))


@pytest.mark.parametrize("lens", [[1], [5], [333], [7, 9000], [20011]], ids=str)
@pytest.mark.parametrize("hq,hkv,d", [(8, 8, 128), (16, 2, 64), (32, 2, 128), (16, 1, 128), (1, 1, 64)])
def test_cache_attention_split_over_blocks(api, lens, hq, hkv, d):
    """Few rows: the work of a sequence is cut into parts that are joined."""
    page = 64
    pages = Pages(lens, hkv, d, page, 29)
    q = torch.randn(len(lens), hq, d, generator=torch.Generator("cuda").manual_seed(31), device="cuda").half()
    got = api.pd_attn_cache(q, *pages.tensors(), i32(lens), pages.block_table, 0.05)
    check_cache(got, q, pages, lens, 0.05, torch.float16)
    assert torch.equal(got, api.pd_attn_cache(q, *pages.tensors(), i32(lens), pages.block_table, 0.05))


def test_cache_attention_many_short_sequences(api):
    rng = np.random.default_rng(37)
    lens = rng.integers(0, 90, 700).tolist()  # more sequences than threads in a block
    pages = Pages(lens, 2, 64, 16, 41)
    q = torch.randn(len(lens), 4, 64, generator=torch.Generator("cuda").manual_seed(1), device="cuda").bfloat16()
    got = api.pd_attn_cache(q, *pages.tensors(), i32(lens), pages.block_table)
    check_cache(got, q, pages, lens, 64 ** -0.5, torch.bfloat16)


def test_cache_attention_strides_and_queries_of_any_size(api):
    lens = [100, 40, 3]
    pages = Pages(lens, 2, 64, 32, 43)
    wide = torch.randn(3, 9, 72, generator=torch.Generator("cuda").manual_seed(2), device="cuda").bfloat16()
    q = wide[:, 1:9, 8:]
    want = api.pd_attn_cache(q.contiguous(), *pages.tensors(), i32(lens), pages.block_table)
    big = torch.full((3, 10, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    api.pd_attn_cache(q, *pages.tensors(), i32(lens), pages.block_table, out=big[:, 1:9])
    assert torch.equal(big[:, 1:9], want) and bool((big[:, 0] == 5.0).all() and (big[:, 9] == 5.0).all())
    for factor in (2.0 ** -100, 2.0 ** 90):  # far outside binary16: only the exponent of a query moves
        got = api.pd_attn_cache(q * factor, *pages.tensors(), i32(lens), pages.block_table, 64 ** -0.5 / factor)
        assert torch.equal(got, want)
    zero = api.pd_attn_cache(torch.zeros_like(q), *pages.tensors(), i32(lens), pages.block_table)
    check_cache(zero, torch.zeros_like(q), pages, lens, 64 ** -0.5, torch.bfloat16)


def test_cache_attention_scales_of_very_different_size(api):
    lens = [400, 65]
    pages = Pages(lens, 2, 128, 16, 47)
    factor = torch.from_numpy(10.0 ** pages.rng.integers(-6, 5, tuple(pages.v_scale.shape))).float().cuda()
    pages.v_scale *= factor
    pages.v_scale[pages.table[0, 3]] = 0.0
    pages.k_scale[pages.table[0, 5]] = 0.0
    q = torch.randn(2, 6, 128, generator=torch.Generator("cuda").manual_seed(3), device="cuda").half()
    got = api.pd_attn_cache(q.bfloat16(), *pages.tensors(), i32(lens), pages.block_table)
    check_cache(got, q.bfloat16(), pages, lens, 128 ** -0.5, torch.bfloat16)


def test_cache_attention_non_finite_pages(api):
    lens = [100, 100]
    pages = Pages(lens, 2, 64, 32, 53)
    q = torch.randn(2, 4, 64, generator=torch.Generator("cuda").manual_seed(4), device="cuda").half()
    clean = api.pd_attn_cache(q, *pages.tensors(), i32(lens), pages.block_table)
    pages.v_scale[pages.table[0, 1], 1] = float("nan")
    got = api.pd_attn_cache(q, *pages.tensors(), i32(lens), pages.block_table)
    assert bool(torch.isnan(got[0, 2:].float()).all())
    assert torch.equal(got[0, :2], clean[0, :2]) and torch.equal(got[1], clean[1])


def test_cache_attention_bad_indices_are_reported(api):
    lens = [100, 40]
    pages = Pages(lens, 2, 64, 32, 59)
    q = torch.randn(2, 4, 64, generator=torch.Generator("cuda").manual_seed(6), device="cuda").half()
    clean = api.pd_attn_cache(q, *pages.tensors(), i32(lens), pages.block_table)
    for entry in (-1, pages.n_pages, 2 ** 31 - 1):
        table = pages.block_table.clone()
        table[0, 2] = entry
        got = api.pd_attn_cache(q, *pages.tensors(), i32(lens), table)
        assert api.pd_device_status(api.attn_workspace()) == 8
        assert torch.equal(got[1], clean[1])
    for bad in (-5, pages.width * 32 + 1):
        got = api.pd_attn_cache(q, *pages.tensors(), i32([bad, 40]), pages.block_table.clamp(min=0))
        assert api.pd_device_status(api.attn_workspace()) == 8
        # another length of one sequence moves the places where the others are cut: right, but not the same bits
        want = Pages([100, 40], 2, 64, 32, 59)
        want.table = want.table[1:]
        check_cache(got[1:], q[1:], want, [40], 64 ** -0.5, torch.float16)


def test_cache_offsets_past_32_bits(api):
    """The last pages of a cache of more than 2^32 bytes."""
    hkv, d, page = 8, 128, 64
    n_pages = 2 ** 32 // (hkv * d * page) + 40
    codes = [torch.empty(n_pages, hkv, page, d, dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(n_pages, hkv, dtype=torch.float32, device="cuda") for _ in range(2)]
    gen = torch.Generator("cuda").manual_seed(61)
    k, v = (torch.randn(150, hkv, d, generator=gen, device="cuda").half() for _ in range(2))
    q = torch.randn(1, 16, d, generator=gen, device="cuda").half()
    table = i32([[n_pages - 1, n_pages - 30, n_pages - 7]])
    api.pd_kv_append(k, v, *codes, *scales, offsets([150]), i32([150]), table)
    got = api.pd_attn_cache(q, *codes, *scales, i32([150]), table)
    small = [torch.zeros(3, hkv, page, d, dtype=torch.int8, device="cuda") for _ in range(2)] + [torch.zeros(3, hkv, device="cuda") for _ in range(2)]
    api.pd_kv_append(k, v, *small, offsets([150]), i32([150]), i32([[2, 0, 1]]))
    assert torch.equal(got, api.pd_attn_cache(q, *small, i32([150]), i32([[2, 0, 1]])))
    assert api.pd_device_status(api.attn_workspace()) == 0


# ------------------------------------------------------------------ appending
def check_append(api, held, new, hkv, d, page, dtype, seed, amplitude=1.0):
    total = [a + b for a, b in zip(held, new)]
    pages = Pages(total, hkv, d, page, seed)
    gen = torch.Generator("cuda").manual_seed(seed)
    kv = (amplitude * torch.randn(max(sum(new), 1), 2 * hkv + 1, d, generator=gen, device="cuda")).to(dtype)[:sum(new)]
    k, v = kv[:, :hkv], kv[:, hkv + 1:]
    before = pages.host()
    out = [torch.full((sum(new), hkv, d), 9.0, dtype=dtype, device="cuda") for _ in range(2)]
    api.pd_kv_append(k, v, *pages.tensors(), offsets(new), i32(total), pages.block_table, *out)
    assert api.pd_device_status(api.attn_workspace()) == 0
    after = pages.host()
    for x, codes0, scale0, codes1, scale1, values in ((f64(k), before[0], before[2], after[0], after[2], out[0]), (f64(v), before[1], before[3], after[1], after[3], out[1])):
        want_codes, want_scale = codes0.astype(np.int64), scale0.astype(np.float64)
        orc.kv_append(x, want_codes, want_scale, held, new, pages.table)
        seen = np.isfinite(want_scale)
        assert np.array_equal(np.isfinite(scale1), seen)
        assert np.all(np.abs(scale1[seen] - want_scale[seen]) <= 2.0 ** -23 * want_scale[seen])
        # every code within half a step of what it has to stand for
        at, slots = 0, np.zeros(codes1.shape[:3:2], dtype=bool)
        for b, (h, m) in enumerate(zip(held, new)):
            for pos in range(h // page * page if m else 0, h + m if m else 0):
                p, s = pages.table[b][pos // page], pos % page
                slots[p, s] = True
                step = want_scale[p]
                goal = x[at + pos - h] if pos >= h else codes0[p, :, s].astype(np.float64) * (scale0[p].astype(np.float64))[:, None]
                got = codes1[p, :, s].astype(np.float64)
                assert np.all(np.abs(got * step[:, None] - goal) <= (0.5 + 2.3e-5) * step[:, None] + 1e-300), (b, pos)
                if pos >= h:
                    val = f64(values[at + pos - h])
                    assert np.all(np.abs(val - got * step[:, None]) <= (UNIT[dtype] + 2.0 ** -22) * np.abs(val) + 2.0 ** -25 * (dtype == torch.float16))
            at += m
        where = np.broadcast_to(~slots[:, None, :, None], codes1.shape)
        assert np.array_equal(codes1[where], codes0[where])  # nothing else is written
    return pages


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hkv,d,page", [(2, 128, 64), (1, 64, 16), (3, 64, 128), (2, 128, 128), (2, 128, 16), (1, 64, 32)])
def test_append_matches_the_definition(api, hkv, d, page, dtype):
    check_append(api, [0, 5, page - 1, page, 3 * page + 2, 17, 0], [2 * page + 3, page, 1, 1, 0, 2 * page, 1], hkv, d, page, dtype, 67)


def test_append_single_tokens(api):
    """One token for each of many sequences, with and without growth of the scale."""
    rng = np.random.default_rng(71)
    for amplitude in (0.01, 1.0, 100.0):
        check_append(api, rng.integers(0, 70, 300).tolist(), [1] * 300, 2, 64, 32, torch.float16, 73, amplitude)


def test_append_zeros_tiny_and_non_finite_values(api):
    page, d = 16, 64
    for dtype in TYPES:
        codes = [torch.full((4, 1, page, d), 99, dtype=torch.int8, device="cuda") for _ in range(2)]
        scales = [torch.full((4, 1), 3.0, device="cuda") for _ in range(2)]
        k, v = torch.zeros(40, 1, d, dtype=dtype, device="cuda"), torch.ones(40, 1, d, dtype=dtype, device="cuda")
        if dtype == torch.bfloat16:
            k[16:32] = 1e-38  # a scale below 2^-120
        v[20, 0, 3], v[35, 0, 4] = float("inf"), float("nan")
        values = [torch.empty_like(k) for _ in range(2)]
        table = i32([[2, 0, 3]])
        api.pd_kv_append(k, v, *codes, *scales, offsets([40]), i32([40]), table, *values)
        assert not codes[0][2].any() and not codes[0][0].any() and not values[0].float()[:16].any()
        assert float(scales[0][2]) == 0.0 and bool((codes[0][1] == 99).all()) and float(scales[0][1]) == 3.0
        assert bool((values[1][:16] == 1).all()) and bool(torch.isinf(scales[1][0]).all()) and bool(torch.isnan(scales[1][3]).all())
        q = torch.ones(1, 1, d, dtype=dtype, device="cuda")
        assert bool(torch.isnan(api.pd_attn_cache(q, *codes, *scales, i32([40]), table).float()).all())
        assert bool((api.pd_attn_cache(q, *codes, *scales, i32([16]), table) == 1).all())


def test_append_in_place_values_and_bad_indices(api):
    page, d = 32, 128
    gen = torch.Generator("cuda").manual_seed(79)
    k, v = (torch.randn(50, 2, d, generator=gen, device="cuda").half() for _ in range(2))
    def fresh():
        return [torch.zeros(4, 2, page, d, dtype=torch.int8, device="cuda") for _ in range(2)] + [torch.zeros(4, 2, device="cuda") for _ in range(2)]
    one, two = fresh(), fresh()
    values = [torch.empty_like(k), torch.empty_like(v)]
    table = i32([[1, 3]])
    api.pd_kv_append(k, v, *one, offsets([50]), i32([50]), table, *values)
    k2, v2 = k.clone(), v.clone()
    api.pd_kv_append(k2, v2, *two, offsets([50]), i32([50]), table, k2, v2)
    assert torch.equal(k2, values[0]) and torch.equal(v2, values[1]) and all(torch.equal(a, b) for a, b in zip(one, two))
    for cu, lens, tab in (([0, 51], [51], [[1, 3]]), ([0, 50], [49], [[1, 3]]), ([0, 50], [50], [[1, 4]]), ([0, 50], [50], [[-1, 3]]), ([0, 50], [70], [[1, 3]])):
        api.pd_kv_append(k, v, *fresh(), i32(cu), i32(lens), i32(tab))
        assert api.pd_device_status(api.attn_workspace()) == 8, (cu, lens, tab)


def test_decode_steps_on_their_own_streams(api):
    """Append and attention of several independent layers on four streams give what they give alone."""
    lens, hq, hkv, d, page = [70, 200, 5], 8, 2, 128, 16
    rigs = []
    for i in range(4):
        gen = torch.Generator("cuda").manual_seed(83 + i)
        pages = Pages([n + 1 for n in lens], hkv, d, page, 89 + i)
        rigs.append((pages, torch.randn(3, hq + 2 * hkv, d, generator=gen, device="cuda").bfloat16()))
    after, cu = i32([n + 1 for n in lens]), offsets([1, 1, 1])

    def step(pages, x):
        api.pd_kv_append(x[:, hq:hq + hkv], x[:, hq + hkv:], *pages.tensors(), cu, after, pages.block_table)
        return api.pd_attn_cache(x[:, :hq], *pages.tensors(), after, pages.block_table)

    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in rigs], []
    for s, (pages, x) in zip(streams, rigs):
        with torch.cuda.stream(s):
            outs.append([step(pages, x) for _ in range(5)])  # appending the same tokens again changes nothing
    torch.cuda.synchronize()
    for (pages, x), got in zip(rigs, outs):
        want = step(pages, x)
        assert all(torch.equal(want, o) for o in got)


def test_binding_refusals(api):
    lens = [20]
    q, k, v = prompt_inputs(lens, 4, 2, 64, torch.float16, 97)
    pages = Pages(lens, 2, 64, 16, 101)
    cu, n = offsets(lens), i32(lens)
    with pytest.raises(ValueError):
        api.pd_attn_prompt(q, k[:10], v[:10], cu)
    with pytest.raises(TypeError):
        api.pd_attn_prompt(q, k.float(), v, cu)
    with pytest.raises(TypeError):
        api.pd_attn_prompt(q, k, v, cu.long())
    with pytest.raises(ValueError):
        api.pd_attn_prompt(q.transpose(1, 2).contiguous().transpose(1, 2), k, v, cu)
    with pytest.raises(api.PdError):
        api.pd_attn_prompt(q[:, :3], k, v, cu)
    with pytest.raises(api.PdError):
        api.pd_attn_prompt(q, k[:, :1].expand(-1, 2, -1), v, cu)  # broadcast heads
    with pytest.raises(ValueError):
        api.pd_attn_cache(q[:1, :, :32], *pages.tensors(), n, pages.block_table)
    with pytest.raises(TypeError):
        api.pd_attn_cache(q[:1], pages.k_codes.to(torch.uint8), *pages.tensors()[1:], n, pages.block_table)
    with pytest.raises(ValueError):
        api.pd_attn_cache(q[:2], *pages.tensors(), n, pages.block_table)
    with pytest.raises(ValueError):
        api.pd_kv_append(k, v, *pages.tensors(), cu, n, pages.block_table.repeat(2, 1))
    with pytest.raises(ValueError):
        api.pd_kv_append(k, v, *pages.tensors(), cu, n, pages.block_table, k_values=torch.empty(20, 2, 32, dtype=torch.float16, device="cuda"))
