"""fp64 definitions of the attention operators (prompt attention, the 8-bit paged cache, attention over it) in numpy: plain
loops over sequences and heads.  Test infrastructure only."""
import numpy as np


def softmax_weights(scores):
    """Weights of one query over the scores of the tokens that it attends to."""
    e = np.exp(scores - scores.max())
    return e / e.sum()


def attn_prompt(q, k, v, lens, scale):
    """q [T, Hq, d], k and v [T, Hkv, d] (fp64), lens: tokens of each sequence in order.  Token i attends to 0 .. i."""
    out = np.zeros_like(q)
    group = q.shape[1] // k.shape[1]
    at = 0
    for n in lens:
        for h in range(q.shape[1]):
            for i in range(n):
                s = k[at:at + i + 1, h // group] @ q[at + i, h] * scale
                out[at + i, h] = softmax_weights(s) @ v[at:at + i + 1, h // group]
        at += n
    return out


def kv_append(x, codes, scale, lens_before, lens_new, table):
    """Quantises x [T, H, d] into codes [pages, H, page, d] (int64) and scale [pages, H] (fp64), both changed in place.
    Returns the values that the new codes stand for [T, H, d]."""
    page = codes.shape[2]
    values = np.zeros_like(x)
    at = 0
    for b, (held, new) in enumerate(zip(lens_before, lens_new)):
        pos = held
        while pos < held + new:
            p, lo = table[b][pos // page], pos % page
            n = min(page - lo, held + new - pos)
            for h in range(x.shape[1]):
                y = x[at:at + n, h]
                s_old = scale[p, h] if lo else 0.0
                s_new = max(s_old, np.abs(y).max() / 127)
                if s_new > 0:
                    codes[p, h, :lo] = np.rint(codes[p, h, :lo] * (s_old / s_new))
                    codes[p, h, lo:lo + n] = np.rint(y / s_new)
                else:
                    codes[p, h, lo:lo + n] = 0
                scale[p, h] = s_new
                values[at:at + n, h] = codes[p, h, lo:lo + n] * s_new
            at, pos = at + n, pos + n
    return values


def attn_cache(q, k_codes, v_codes, k_scale, v_scale, lens, table, scale):
    """q [B, Hq, d] (fp64) over the cache; zeros for an empty sequence."""
    out = np.zeros_like(q)
    group = q.shape[1] // k_codes.shape[1]
    page = k_codes.shape[2]
    for b, n in enumerate(lens):
        for h in range(q.shape[1] if n else 0):
            pages = [table[b][i] for i in range(-(-n // page))]
            k = np.concatenate([k_codes[p, h // group].astype(np.float64) * float(k_scale[p, h // group]) for p in pages])[:n]
            v = np.concatenate([v_codes[p, h // group].astype(np.float64) * float(v_scale[p, h // group]) for p in pages])[:n]
            out[b, h] = softmax_weights(k @ q[b, h] * scale) @ v
    return out


def rope(x, positions, inv_freq, axes, interleaved, inverse=False):
    """x [T, heads, d] (fp64), positions [n_axes, T], inv_freq [pairs], axes [pairs]: each pair of each token by itself."""
    out = x.copy()
    pairs = len(inv_freq)
    for t in range(x.shape[0]):
        for i in range(pairs):
            a = float(positions[axes[i]][t]) * float(inv_freq[i]) * (-1 if inverse else 1)
            p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
            out[t, :, p] = x[t, :, p] * np.cos(a) - x[t, :, q] * np.sin(a)
            out[t, :, q] = x[t, :, p] * np.sin(a) + x[t, :, q] * np.cos(a)
    return out


def attn_chunk(q, k_codes, v_codes, k_scale, v_scale, lens, new, table, scale):
    """q [T, Hq, d] (fp64): the last new[b] of the lens[b] tokens of each sequence, which are all in the cache."""
    out = np.zeros_like(q)
    at = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        for i in range(m):
            one = attn_cache(q[at + i:at + i + 1], k_codes, v_codes, k_scale, v_scale, [n - m + i + 1], table[b:b + 1], scale)
            out[at + i] = one[0]
        at += m
    return out
