"""CPU-side checks of the attention operators: every refusal happens on the host before a launch, and the fp64 definitions
that the GPU tests compare with agree with independent forms."""
import ctypes

import numpy as np
import pytest

from oracle import pd_oracle_attn as orc

A = 0x10000  # aligned, never dereferenced
INVALID, SHAPE, ALIGN, WS = 1, 2, 3, 4


@pytest.fixture(scope="module")
def api():
    from paper_2512_19720_b200 import build
    build.build()
    from paper_2512_19720_b200 import api
    return api


def call(fn, spec, **change):
    args = dict(spec)
    unknown = set(change) - set(args)
    assert not unknown, unknown
    args.update(change)
    return fn(*args.values())


PROMPT = dict(q=A, q_t=1024, q_h=128, k=A, k_t=1024, k_h=128, v=A, v_t=1024, v_h=128, cu=A, n_seqs=2, n_tokens=10, q_heads=8, kv_heads=8,
              head_dim=128, scale=0.1, out=A, out_t=1024, out_h=128, ws=A, ws_bytes=1 << 30, stream=None)
APPEND = dict(k=A, k_t=1024, k_h=128, v=A, v_t=1024, v_h=128, cu=A, n_seqs=2, n_tokens=10, kv_heads=8, head_dim=128, k_codes=A, v_codes=A,
              k_scale=A, v_scale=A, n_pages=4, page=16, seq_lens=A, table=A, table_stride=4, table_width=4, k_values=None, v_values=None, ws=A,
              ws_bytes=1 << 30, stream=None)
CACHE = dict(q=A, q_t=1024, q_h=128, n_seqs=2, q_heads=8, kv_heads=8, head_dim=128, scale=0.1, k_codes=A, v_codes=A, k_scale=A, v_scale=A,
             n_pages=4, page=16, seq_lens=A, table=A, table_stride=4, table_width=4, out=A, out_t=1024, out_h=128, ws=A, ws_bytes=1 << 30,
             stream=None)


@pytest.mark.parametrize("suffix", ["", "_bf16"])
def test_refusals(api, suffix):
    lib = api.lib
    before = lib.pd_launch_count()
    for name, spec in (("pd_attn_prompt", PROMPT), ("pd_kv_append", APPEND), ("pd_attn_cache", CACHE)):
        fn = getattr(lib, name + suffix)
        for pointer in ("q", "k", "v", "out", "cu", "k_codes", "v_codes", "k_scale", "v_scale", "seq_lens", "table"):
            if pointer in spec:
                assert call(fn, spec, **{pointer: None}) == INVALID, (name, pointer)
        for pointer in ("q", "k", "v", "out", "k_codes", "v_codes"):
            if pointer in spec:
                assert call(fn, spec, **{pointer: A + 8}) == ALIGN, (name, pointer)
        for pointer in ("cu", "k_scale", "seq_lens", "table"):
            if pointer in spec:
                assert call(fn, spec, **{pointer: A + 2}) == ALIGN, (name, pointer)
        for view in ("q", "k", "v", "out"):
            if view in spec:
                assert call(fn, spec, **{view + "_t": 1028}) == ALIGN
                assert call(fn, spec, **{view + "_h": 132}) == ALIGN
                assert call(fn, spec, **{view + "_t": 0}) == INVALID    # a broadcast tensor
                assert call(fn, spec, **{view + "_h": 64}) == INVALID   # heads that overlap
        assert call(fn, spec, n_seqs=0) == INVALID
        assert call(fn, spec, head_dim=96) == SHAPE
        assert call(fn, spec, kv_heads=0) == INVALID
        if "q_heads" in spec:
            assert call(fn, spec, q_heads=12) == INVALID
            assert call(fn, spec, scale=float("nan")) == INVALID
        if "n_tokens" in spec:
            assert call(fn, spec, n_tokens=-1) == INVALID
            assert call(fn, spec, n_tokens=1 << 40) == SHAPE
        if "page" in spec:
            assert call(fn, spec, page=48) == SHAPE
            assert call(fn, spec, n_pages=0) == INVALID
            assert call(fn, spec, table_width=0) == INVALID
            assert call(fn, spec, table_stride=3) == INVALID
        assert call(fn, spec, ws=None) == WS
        assert call(fn, spec, ws=A + 64) == WS
        assert call(fn, spec, ws_bytes=api.workspace_bytes(api.OP_ATTN) - 1) == WS
    assert call(getattr(lib, "pd_kv_append" + suffix), APPEND, k_values=A + 8) == ALIGN
    # nothing to do: no launch, and empty tensors may have no address
    assert call(getattr(lib, "pd_attn_prompt" + suffix), PROMPT, n_tokens=0, q=None, k=None, v=None, out=None) == 0
    assert call(getattr(lib, "pd_kv_append" + suffix), APPEND, n_tokens=0, k=None, v=None) == 0
    assert lib.pd_launch_count() == before


def test_status_and_workspace(api):
    assert "out of range" in api.status_string(8)
    assert api.workspace_bytes(api.OP_ATTN) > 256 and api.workspace_bytes(api.OP_ATTN) % 16 == 0


def test_binding_refuses_cpu_tensors(api):
    import torch
    x = torch.zeros(4, 2, 64, dtype=torch.float16)
    cu = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(TypeError):
        api.pd_attn_prompt(x, x, x, cu)
    with pytest.raises(TypeError):
        api.pd_attn_cache(x, x, x, x, x, cu, cu)


def test_prompt_definition_against_a_masked_matrix_form():
    rng = np.random.default_rng(1)
    lens, hq, hkv, d = [5, 0, 1, 9], 4, 2, 8
    q, k, v = rng.normal(size=(15, hq, d)), rng.normal(size=(15, hkv, d)), rng.normal(size=(15, hkv, d))
    out = orc.attn_prompt(q, k, v, lens, 0.3)
    seq = np.repeat(np.arange(len(lens)), lens)
    see = (seq[:, None] == seq[None, :]) & (np.arange(15)[None, :] <= np.arange(15)[:, None])
    for h in range(hq):
        e = np.where(see, np.exp(q[:, h] @ k[:, h // 2].T * 0.3), 0)
        assert np.allclose(out[:, h], e / e.sum(1, keepdims=True) @ v[:, h // 2], atol=1e-12)
    # the first token of a sequence attends to itself alone
    assert np.allclose(out[5], np.repeat(v[5], 2, axis=0))


def test_cache_definitions_closed_forms():
    rng = np.random.default_rng(2)
    codes, scale = np.zeros((6, 2, 16, 8), dtype=np.int64), np.zeros((6, 2))
    x = rng.normal(size=(40, 2, 8))
    table = [[3, 1, 4]]
    values = orc.kv_append(x, codes, scale, [0], [40], table)
    assert np.abs(codes).max() == 127 and np.all(np.abs(values - x) <= 0.5 * np.repeat(scale[[3, 1, 4]], [16, 16, 8], axis=0)[:, :, None] + 1e-12)
    # a cache written at once or token by token holds the same values up to what rounding again costs: half a step of the final scale at each growth
    codes1, scale1 = np.zeros_like(codes), np.zeros_like(scale)
    for i in range(40):
        orc.kv_append(x[i:i + 1], codes1, scale1, [i], [1], table)
    assert np.allclose(scale1[[3, 1, 4]], scale[[3, 1, 4]])
    whole, pieces = codes[3] * scale[3][:, None, None], codes1[3] * scale1[3][:, None, None]
    assert np.abs(whole - pieces).max() <= 16 * 0.5 * scale[3].max()
    # one token: its value; equal keys: the mean
    q = rng.normal(size=(1, 4, 8))
    v_at = lambda i: codes[table[0][i // 16], :, i % 16] * scale[table[0][i // 16]][:, None]  # noqa: E731
    out = orc.attn_cache(q, codes, codes, scale, scale, [1], table, 0.5)
    assert np.allclose(out[0], np.repeat(v_at(0), 2, axis=0))
    flat = np.zeros_like(codes)
    out = orc.attn_cache(q, flat, codes, scale, scale, [37], table, 0.5)
    assert np.allclose(out[0], np.repeat(np.mean([v_at(i) for i in range(37)], axis=0), 2, axis=0))
    assert not orc.attn_cache(q, flat, codes, scale, scale, [0], table, 0.5).any()
