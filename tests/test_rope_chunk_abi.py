"""CPU-side checks of the calls for positions and pieces (pd_rope, pd_kv_append_rope, pd_attn_chunk): every refusal happens on the host before a
launch, and the fp64 definitions that the GPU tests compare with agree with independent forms."""
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


TURN = dict(positions=A, axis_stride=10, n_axes=3, axes=A, inv_freq=A, pairs=64, interleaved=0)
CACHE = dict(k_codes=A, v_codes=A, k_scale=A, v_scale=A, n_pages=4, page=16, seq_lens=A, table=A, table_stride=4, table_width=4)
END = dict(ws=A, ws_bytes=1 << 30, stream=None)
ROPE = dict(q=A, q_t=1024, q_h=128, k=A, k_t=1024, k_h=128, **TURN, inverse=0, n_tokens=10, q_heads=8, k_heads=8, head_dim=128, q_out=A, q_out_t=1024, q_out_h=128,
            k_out=A, k_out_t=1024, k_out_h=128, **END)
APPEND = dict(q=A, q_t=1024, q_h=128, k=A, k_t=1024, k_h=128, v=A, v_t=1024, v_h=128, cu=A, n_seqs=2, n_tokens=10, q_heads=8, kv_heads=8, head_dim=128, **TURN, **CACHE,
              q_out=A, q_out_t=1024, q_out_h=128, k_values=None, v_values=None, **END)
CHUNK = dict(q=A, q_t=1024, q_h=128, cu=A, n_seqs=2, n_tokens=10, max_new=0, q_heads=8, kv_heads=8, head_dim=128, scale=0.1, **CACHE, out=A, out_t=1024, out_h=128, **END)


@pytest.mark.parametrize("suffix", ["", "_bf16"])
def test_refusals(api, suffix):
    lib = api.lib
    before = lib.pd_launch_count()
    for name, spec, op in (("pd_rope", ROPE, api.OP_ATTN), ("pd_kv_append_rope", APPEND, api.OP_ATTN), ("pd_attn_chunk", CHUNK, api.OP_ATTN_CHUNK)):
        fn = getattr(lib, name + suffix)
        for pointer in ("q", "k", "v", "q_out", "k_out", "out", "cu", "inv_freq", "k_codes", "v_codes", "k_scale", "v_scale", "seq_lens", "table"):
            if pointer in spec:
                assert call(fn, spec, **{pointer: None}) == INVALID, (name, pointer)
        for pointer in ("q", "k", "v", "q_out", "k_out", "out", "k_codes", "v_codes"):
            if pointer in spec:
                assert call(fn, spec, **{pointer: A + 8}) == ALIGN, (name, pointer)
        for pointer in ("cu", "positions", "axes", "inv_freq", "k_scale", "seq_lens", "table"):
            if pointer in spec:
                assert call(fn, spec, **{pointer: A + 2}) == ALIGN, (name, pointer)
        for view in ("q", "k", "v", "q_out", "k_out", "out"):
            if view + "_t" in spec:
                assert call(fn, spec, **{view + "_t": 1028}) == ALIGN
                assert call(fn, spec, **{view + "_h": 132}) == ALIGN
                assert call(fn, spec, **{view + "_t": 0}) == INVALID    # a broadcast tensor
                assert call(fn, spec, **{view + "_h": 64}) == INVALID   # heads that overlap
        assert call(fn, spec, head_dim=96) == SHAPE
        assert call(fn, spec, n_tokens=-1) == INVALID
        assert call(fn, spec, n_tokens=1 << 40) == SHAPE
        if "n_seqs" in spec:
            assert call(fn, spec, n_seqs=0) == INVALID
            assert call(fn, spec, kv_heads=0) == INVALID
        if "page" in spec:
            assert call(fn, spec, page=48) == SHAPE
            assert call(fn, spec, n_pages=0) == INVALID
            assert call(fn, spec, table_width=0) == INVALID
            assert call(fn, spec, table_stride=3) == INVALID
        if "pairs" in spec:
            assert call(fn, spec, pairs=0) == INVALID
            assert call(fn, spec, pairs=12) == SHAPE
            assert call(fn, spec, pairs=72) == SHAPE          # more than the head has
            assert call(fn, spec, interleaved=2) == INVALID
            assert call(fn, spec, n_axes=0) == INVALID
            assert call(fn, spec, axes=None) == INVALID       # three axes and no word on which pair turns with which
            assert call(fn, spec, axis_stride=9) == INVALID   # rows that overlap
        assert call(fn, spec, ws=None) == WS
        assert call(fn, spec, ws=A + 64) == WS
        assert call(fn, spec, ws_bytes=api.workspace_bytes(op) - 1) == WS
    rope, append, chunk = (getattr(lib, n + suffix) for n in ("pd_rope", "pd_kv_append_rope", "pd_attn_chunk"))
    assert call(rope, ROPE, positions=None, axes=None, n_axes=1) == INVALID         # a token's place is not known here
    assert call(append, APPEND, positions=None) == INVALID                          # a place in a sequence has one axis
    assert call(append, APPEND, k_values=A + 8) == ALIGN
    assert call(append, APPEND, q_heads=-1) == INVALID
    assert call(rope, ROPE, q_heads=0) == INVALID
    assert call(chunk, CHUNK, q_heads=12) == INVALID
    assert call(chunk, CHUNK, scale=float("inf")) == INVALID
    assert call(chunk, CHUNK, max_new=-1) == INVALID
    assert call(chunk, CHUNK, n_pages=(1 << 31) // 8) == SHAPE and call(chunk, CHUNK, n_pages=1 << 60) == SHAPE
    # nothing to do: no launch, and empty tensors may have no address
    assert call(rope, ROPE, n_tokens=0, q=None, k=None, q_out=None, k_out=None, positions=None) == 0
    assert call(append, APPEND, n_tokens=0, q=None, k=None, v=None, q_out=None, positions=None) == 0
    assert call(chunk, CHUNK, n_tokens=0, q=None, out=None) == 0
    assert lib.pd_launch_count() == before


def test_binding_refusals(api):
    import torch
    x = torch.zeros(4, 2, 64, dtype=torch.float16)
    i = torch.zeros(4, dtype=torch.int32)
    f = torch.ones(32)
    with pytest.raises(TypeError):
        api.pd_rope(x, x, i, f)
    with pytest.raises(TypeError):
        api.pd_kv_append_rope(x, x, x, x, x, x, x, i, i, i, f)
    with pytest.raises(TypeError):
        api.pd_attn_chunk(x, x, x, x, x, i, i, i)


def test_workspaces(api):
    assert api.workspace_bytes(api.OP_ATTN_CHUNK) > api.workspace_bytes(api.OP_ATTN) and api.workspace_bytes(api.OP_ATTN_CHUNK) % 16 == 0


def test_rotation_definition_against_complex_numbers():
    rng = np.random.default_rng(1)
    x, positions, freq, axes = rng.normal(size=(5, 3, 20)), rng.integers(-9, 9, (2, 5)), rng.normal(size=8), [0, 1, 1, 0, 0, 1, 0, 1]
    t = np.stack([positions[axes[i]] * freq[i] for i in range(8)], axis=1)[:, None]
    for interleaved in (False, True):
        y = orc.rope(x, positions, freq, axes, interleaved)
        a, b = (slice(0, 16, 2), slice(1, 16, 2)) if interleaved else (slice(0, 8), slice(8, 16))
        z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * t)
        assert np.allclose(y[..., a], z.real, atol=1e-12) and np.allclose(y[..., b], z.imag, atol=1e-12)
        assert np.array_equal(y[..., 16:], x[..., 16:])
        assert np.allclose(orc.rope(y, positions, freq, axes, interleaved, inverse=True), x, atol=1e-12)
    # scores depend on the distance of two positions alone
    q, k = rng.normal(size=(1, 1, 16)), rng.normal(size=(1, 1, 16))
    score = lambda p, r: float((orc.rope(q, [[p]], freq, [0] * 8, False) * orc.rope(k, [[r]], freq, [0] * 8, False)).sum())  # noqa: E731
    assert np.isclose(score(3, 1), score(103, 101), atol=1e-9)


def test_piece_definition_against_a_masked_matrix_form():
    rng = np.random.default_rng(2)
    page, table = 4, np.array([[2, 0, 3], [1, 4, -1]])
    codes = [rng.integers(-127, 128, (5, 2, page, 8)) for _ in range(2)]
    scales = [rng.uniform(0.5, 2, (5, 2)) / 100 for _ in range(2)]
    lens, new = [11, 6], [3, 6]
    q = rng.normal(size=(9, 4, 8))
    out = orc.attn_chunk(q, *codes, *scales, lens, new, table, 0.4)
    at = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        p = table[b, :-(-n // page)]
        k, v = ((c[p] * s[p][:, :, None, None]).transpose(1, 0, 2, 3).reshape(2, -1, 8)[:, :n] for c, s in zip(codes, scales))
        see = np.arange(n)[None, :] <= np.arange(n - m, n)[:, None]
        for h in range(4):
            e = np.where(see, np.exp(q[at:at + m, h] @ k[h // 2].T * 0.4), 0)
            assert np.allclose(out[at:at + m, h], e / e.sum(1, keepdims=True) @ v[h // 2], atol=1e-12)
        at += m
