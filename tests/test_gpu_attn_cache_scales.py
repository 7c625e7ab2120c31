"""pd_attn_cache where the scales of V fall and rise again by any factor: against the fp64 definition of test_gpu_attn_edges, at its bounds."""
import numpy as np
import pytest
import torch

from test_gpu_attn_edges import Cache, attend, check, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2512_19720_b200 import api
    return api


def check_some(api, cache, q, scale, some):
    got = attend(api, cache, q, scale)
    assert bool(torch.isfinite(got).all())
    part = Cache([cache.lens[b] for b in some], cache.k_codes.shape[1], cache.k_codes.shape[3], cache.page, 0)
    rows = np.concatenate([cache.table[b, :-(-cache.lens[b] // cache.page)] for b in some])
    for name in ("k_codes", "v_codes", "k_scale", "v_scale"):
        setattr(part, name, getattr(cache, name)[rows])
    want, bound = part.definition(f64(q[some]), scale, torch.bfloat16)
    check(got[some], want, bound)


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 128), (12, 1, 64), (2, 2, 64)])
@pytest.mark.parametrize("n_seqs", [3, 700])
def test_scales_at_random_over_the_whole_range(api, n_seqs, hq, hkv, d):
    """Few sequences, whose pages are spread over many warps, and many, whose pages one warp goes through one after another."""
    cache = Cache([16 * 40 + 7] * n_seqs, hkv, d, 16, 3)
    rng = np.random.default_rng(5)
    cache.v_scale[:] = 2.0 ** rng.uniform(-119, 119, cache.v_scale.shape)
    q = (0.3 * torch.randn(n_seqs, hq, d, generator=torch.Generator("cuda").manual_seed(7), device="cuda")).bfloat16()
    check_some(api, cache, q, d ** -0.5, list(range(min(n_seqs, 12))))


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 128), (12, 1, 64)])
@pytest.mark.parametrize("lead", [0.0, 30.0, 150.0])
def test_a_scale_that_rises_again_far_below_the_largest(api, lead, hq, hkv, d):
    """The first pages hold the largest values, and weights that vanish or do not; then the scales fall as far as they go and rise in steps."""
    page, n_seqs = 32, 700
    cache = Cache([8 * page] * n_seqs, hkv, d, page, 11)
    steps = np.array([2.0 ** 100, 2.0 ** -119, 2.0 ** -100, 2.0 ** -60, 2.0 ** -30, 2.0 ** -50, 1.0, 2.0 ** 20], dtype=np.float32)
    cache.v_scale[:] = np.tile(steps, n_seqs)[:, None]
    early = np.arange(8 * n_seqs) % 8 == 0
    cache.k_scale[:] = 2.0 ** -6
    cache.k_codes[early, ..., 0], cache.k_codes[~early, ..., 0] = -64, 64
    q = 0.1 * torch.randn(n_seqs, hq, d, generator=torch.Generator("cuda").manual_seed(13), device="cuda")
    q[..., 0] = lead
    check_some(api, cache, q.bfloat16(), 1.0, [0, 1, 99, n_seqs - 1])
