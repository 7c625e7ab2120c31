"""Measured cases of the operators that turn a block's linears into a decoder's attention when tokens come in pieces: rotary
positions with one or several axes (pd_rope), rotating and appending to the 8-bit paged cache in one call (pd_kv_append_rope) and
attention of several new tokens a sequence over that cache (pd_attn_chunk).

Head layouts are those of the two block shapes that the library's linears are benchmarked on: 32 query and 32 key/value
heads of 128 (q/k/v 4096 x 4096) and 64 query and 8 key/value heads of 128 (q 8192 x 8192, k/v 1024 x 8192), and small
ones with heads of 64.  Batches (64 decode tokens, 4 prompts of 512 tokens) and prompt lengths (up to 8192 tokens) are
the benchmark's too.

Formulas.  Rotation of a token with positions p[a] (one for each axis): pair i of a head, values (x, y), turns by the angle
t = p[axes[i]] * inv_freq[i] to (x cos t - y sin t, x sin t + y cos t).  Pair i is (i, i + pairs) or, interleaved, (2 i, 2 i + 1);
values behind the 2 * pairs first ones of a head stay as they are.
Cache: page p, head g holds codes c (int8) and a scale s, and stands for the values c * s.  Appending to a page:
    s' = max(s of what the page holds, max |new values| / 127),  held codes c' = round(c * s / s'),  new codes = round(x / s')
with the rotated keys, which are not rounded before that.  A page whose first token is among the new ones starts from s = 0.
Pieces: token i of the n new ones of a sequence of (with them) l tokens, query head h, key/value head g = h // (q_heads / kv_heads):
    out[i, h] = sum_j softmax_j(scale * q[i, h] . K[j, g]) V[j, g]  over the tokens j <= l - n + i
"""
import math
import random

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
SMALLEST_SCALE = 2.0 ** -120  # a page whose scale is below this holds zeros


def listed():
    def case(name, kind, dtype, q_heads, kv_heads, head_dim, batch, new, held=(0, 0), lens_seed=1, page=64, rot=None, axes=1, interleaved=False):
        return {"name": name, "kind": kind, "dtype": dtype, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "batch": batch,
                "min_new": new[0], "max_new": new[1], "min_held": held[0], "max_held": held[1], "lens_seed": lens_seed, "page": page,
                "rot": rot or head_dim, "axes": axes, "interleaved": interleaved}
    return [
        # a single short prompt through a small layer, pairs side by side: what counts is the latency of a call
        case("rope_small", "rope", "fp16", 12, 4, 64, 1, (17, 17), interleaved=True),
        # the prompts of the multi-variant batch (4 x 512 tokens), 7B heads
        case("rope_7b_4x512", "rope", "fp16", 32, 32, 128, 4, (512, 512)),
        # a clip of frames with positions in time, height and width, 70B heads
        case("rope_70b_video", "rope", "bf16", 64, 8, 128, 1, (8160, 8160), axes=3),
        # a decode step: each of 64 sequences gets a token, far positions among them, 70B heads
        case("append_70b_step", "append", "bf16", 64, 8, 128, 64, (1, 1), (1, 131000)),
        # the keys and values of the multi-variant batch's prompts go into fresh pages, rotated on the way
        case("append_7b_4x512", "append", "fp16", 32, 32, 128, 4, (512, 512)),
        # the next pieces of inputs with pictures, positions in two axes for half of each head: they go on in the middle of a page
        case("append_70b_pieces", "append", "bf16", 64, 8, 128, 9, (1, 1700), (0, 1000), lens_seed=3, rot=64, axes=2),
        # one user's few drafted tokens behind a short conversation, a small layer: latency again
        case("chunk_small", "chunk", "fp16", 8, 8, 64, 1, (5, 5), (300, 300), page=32),
        # four drafted tokens for each of 64 sequences are looked at together, 70B heads, small pages
        case("chunk_70b_draft", "chunk", "bf16", 64, 8, 128, 64, (4, 4), (200, 8000), page=16),
        # the next 512 tokens of 4 prompts that are read in pieces, 7B heads
        case("chunk_7b_4x512", "chunk", "fp16", 32, 32, 128, 4, (512, 512), (0, 1600), lens_seed=7),
        # pieces of very different lengths in one batch, single tokens among them, 70B heads
        case("chunk_70b_mixed", "chunk", "bf16", 64, 8, 128, 10, (1, 500), (0, 4000), lens_seed=11, page=128),
        # a piece of a long document, 70B heads
        case("chunk_70b_2048", "chunk", "bf16", 64, 8, 128, 1, (2048, 2048), (16384, 16384)),
        # a pass over drafted tokens as it is run: 64 sequences get 1 to 8 tokens each, rotated, appended and attended with, 7B heads
        case("pass_7b_draft", "pass", "fp16", 32, 32, 128, 64, (1, 8), (20, 1000), lens_seed=5),
    ]


def draw(rng):
    kind = rng.choice(["rope", "append", "chunk", "chunk", "pass"])
    q_heads, kv_heads = rng.choice([(8, 8), (32, 32), (64, 8), (32, 8), (12, 4), (16, 1), (40, 8), (5, 5)])
    head_dim = rng.choice([64, 128, 128])
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    if kind in ("rope", "append"):
        batch = log(1, 64)
        most_new, most_held = log(1, max(1, 8160 // batch)), log(1, 4000)
    else:
        batch = log(1, 64)
        most_new, most_held = log(1, 2048 if kind == "chunk" else 64), log(1, 65536)
        most_new = max(1, min(most_new, 8192 // batch))
        # no more work than the largest listed case, and no cache beyond 2 GB
        while q_heads * batch * most_new * (most_held + most_new) > 64 * 2048 * 18432 or batch * kv_heads * (most_held + most_new) > 8_000_000:
            if most_held > most_new:
                most_held //= 2
            else:
                most_new //= 2
    least_new = most_new if rng.random() < 0.4 else rng.randint(0 if batch > 2 and kind == "chunk" else 1, most_new)
    return {"kind": kind, "dtype": rng.choice(["fp16", "bf16"]), "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "batch": batch,
            "min_new": least_new, "max_new": most_new, "min_held": rng.randint(0, most_held), "max_held": most_held, "lens_seed": rng.randrange(1000),
            "page": rng.choice([16, 32, 64, 128]), "rot": rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 4 * 3]), "axes": rng.choice([1, 1, 2, 3]),
            "interleaved": rng.random() < 0.3}


def lengths(case):
    """(tokens that each sequence holds before the call, tokens of the call); one sequence at least has the most new ones."""
    r = random.Random(case["lens_seed"])
    new = [r.randint(case["min_new"], case["max_new"]) for _ in range(case["batch"])]
    new[r.randrange(case["batch"])] = case["max_new"]
    return [r.randint(case["min_held"], case["max_held"]) for _ in new], new


def prepare(case, seed):
    dev, dt = torch.device("cuda"), DTYPES[case["dtype"]]
    gen = torch.Generator(device=dev).manual_seed(seed)
    kind, (held, new) = case["kind"], lengths(case)
    total = [a + b for a, b in zip(held, new)]
    n_new, b, hq, hkv, d = sum(new), case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"]
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=dev, dtype=dt)  # noqa: E731
    # some channels of keys are much larger than others, as they are behind a linear
    channel = 2.0 ** (0.7 * torch.randn(hkv, d, generator=gen, device=dev))
    s = {"case": case, "scale": 1.0 / math.sqrt(d), "most_new": case["max_new"]}
    # queries, keys and values of the new tokens are slices of one fused projection's output, as a user's program has them
    qkv = normal(n_new, hq + 2 * hkv, d)
    s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    s["k"].mul_(channel.to(dt))
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    s["cu_seqlens"] = torch.tensor(cu, dtype=torch.int32, device=dev)
    s["seq_lens"] = torch.tensor(total, dtype=torch.int32, device=dev)  # with the new tokens
    old = torch.tensor(held, device=dev)
    seq_of = torch.repeat_interleave(torch.arange(b, device=dev), torch.tensor(new, device=dev), output_size=n_new)
    in_piece = torch.arange(n_new, device=dev) - s["cu_seqlens"].long()[seq_of]
    pos = old[seq_of] + in_piece
    s["seq_of"], s["in_piece"] = seq_of, in_piece
    # what a model keeps: the frequencies and, where there are several axes, which of them each pair turns with
    pairs = case["rot"] // 2
    s["inv_freq"] = (500000.0 ** (-torch.arange(pairs, device=dev, dtype=torch.float64) / pairs)).float()
    s["axes"] = None if case["axes"] == 1 else (torch.arange(pairs, device=dev) * case["axes"] // pairs).to(torch.int32)
    rows, cols = 20, 34  # patches of a picture
    grid = [old[seq_of] + in_piece // (rows * cols), old[seq_of] + in_piece // cols % rows, old[seq_of] + in_piece % cols]
    s["positions"] = torch.stack([pos] if case["axes"] == 1 else grid[3 - case["axes"]:]).to(torch.int32)
    s["q_out"], s["k_out"], s["v_out"] = torch.empty(n_new, hq, d, dtype=dt, device=dev), *(torch.empty(n_new, hkv, d, dtype=dt, device=dev) for _ in range(2))
    s["out"] = torch.empty(n_new, hq, d, dtype=dt, device=dev)
    if kind == "rope":
        return s
    page = case["page"]
    # a decode step's far positions need no pages between: only what the call touches is there, the rest of the table says so
    first_page = [h // page if kind == "append" else 0 for h in held]
    pages = [-(-t // page) - f for t, f in zip(total, first_page)]
    n_pages = sum(pages) + 8  # a cache has pages that nobody uses
    width = max(max(f + p for f, p in zip(first_page, pages)), 1) + 1
    perm = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32)
    at, first = torch.arange(width, device=dev), torch.tensor([sum(pages[:i]) for i in range(b)], device=dev)
    lo, n_of = torch.tensor(first_page, device=dev), torch.tensor(pages, device=dev)
    there = (at[None, :] >= lo[:, None]) & (at[None, :] < (lo + n_of)[:, None])
    index = torch.where(there, first[:, None] + at[None, :] - lo[:, None], torch.zeros_like(at)[None, :])
    s["block_table"] = table = torch.where(there, perm[index], torch.full((), -1, dtype=torch.int32, device=dev)).contiguous()
    for name, ch in (("k", channel), ("v", torch.ones_like(channel))):
        codes = torch.empty(n_pages, hkv, page, d, dtype=torch.int8, device=dev)
        scale = torch.empty(n_pages, hkv, dtype=torch.float32, device=dev)
        for i in range(0, n_pages, 4096):  # in pieces: the values in 16 bits need not all be there at once
            x = normal(min(4096, n_pages - i), hkv, page, d) * ch[:, None].to(dt)
            amax = x.abs().amax(dim=(2, 3)).float()
            scale[i:i + 4096] = amax / 127
            codes[i:i + 4096] = torch.round(x.float() * (127 / amax)[:, :, None, None]).to(torch.int8)
        s[name + "_codes"], s[name + "_scale"] = codes, scale
    if kind in ("append", "pass"):
        # for the plain form: the pages that the new tokens touch, the page that each of them goes to, and how many tokens each page holds
        touched = there & (at[None, :] >= (old // page)[:, None]) & (torch.tensor(new, device=dev) > 0)[:, None]
        where = touched.nonzero()
        s["touched"] = table[where[:, 0], where[:, 1]].long()
        s["held_in"] = (old[where[:, 0]] - where[:, 1] * page).clamp(min=0, max=page)
        index = torch.zeros(b, width, dtype=torch.long, device=dev)
        index[where[:, 0], where[:, 1]] = torch.arange(len(where), device=dev)
        s["touched_of"], s["slot_of"] = index[seq_of, pos // page], pos % page
    return s


# ---------------------------------------------------------------------------------------------- the plain forms
def plain_rotate(s, x):
    """x [T, heads, d] rotated, in 32 bits; angles in 64, where far positions need them."""
    pairs = s["inv_freq"].numel()
    axes = s["axes"].long() if s["axes"] is not None else torch.zeros(pairs, dtype=torch.long, device=x.device)
    angle = s["positions"].double()[axes].T * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    out = x.float()
    if s["case"]["interleaved"]:
        a, b = out[..., 0:2 * pairs:2], out[..., 1:2 * pairs:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    else:
        a, b = out[..., :pairs], out[..., pairs:2 * pairs]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    return torch.cat((turned, out[..., 2 * pairs:]), dim=-1)


def plain_append(s, x, name):
    codes, scale = s[name + "_codes"], s[name + "_scale"]
    page, touched = codes.shape[2], s["touched"]
    amax = torch.zeros(len(touched), codes.shape[1], device=x.device)
    amax.scatter_reduce_(0, s["touched_of"][:, None].expand(-1, codes.shape[1]), x.abs().amax(dim=2), "amax")
    before = torch.where(s["held_in"][:, None] > 0, scale[touched], torch.zeros_like(amax))
    after = torch.maximum(before, amax / 127)
    inverse = torch.where(after >= SMALLEST_SCALE, 1 / after, torch.zeros_like(after))
    old = codes[touched]
    again = torch.round(old.float() * (before * inverse)[:, :, None, None]).to(torch.int8)
    stays = torch.arange(page, device=x.device)[None, :] >= s["held_in"][:, None]
    codes[touched] = torch.where(stays[:, None, :, None], old, again)
    scale[touched] = after
    fresh = torch.round(x * inverse[s["touched_of"]][:, :, None]).to(torch.int8)
    codes[touched[s["touched_of"]], :, s["slot_of"]] = fresh
    return (fresh.float() * after[s["touched_of"]][:, :, None]).to(s["q"].dtype)


def plain_chunk(s, q):
    c, n, page = s["case"], s["most_new"], s["case"]["page"]
    b, hkv, d = c["batch"], c["kv_heads"], c["head_dim"]
    group = c["q_heads"] // hkv
    cu, lens = s["cu_seqlens"].long(), s["seq_lens"].long()
    at = torch.arange(n, device=q.device)
    count = cu[1:] - cu[:-1]
    index = torch.where(at[None, :] < count[:, None], cu[:-1, None] + at[None, :], torch.zeros_like(at)[None, :])
    qf = (q.float() * s["scale"])[index].view(b, n, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, group * n, d)
    pages = s["block_table"].clamp(min=0).long()
    m = pages.shape[1] * page
    kf = (s["k_codes"][pages].float() * s["k_scale"][pages][..., None, None]).permute(0, 2, 1, 3, 4).reshape(b, hkv, m, d)
    vf = (s["v_codes"][pages].float() * s["v_scale"][pages][..., None, None]).permute(0, 2, 1, 3, 4).reshape(b, hkv, m, d)
    last = (lens - count)[:, None] + at[None, :]
    keep = torch.arange(m, device=q.device)[None, None, :] <= last[:, :, None]
    scores = torch.matmul(qf, kf.transpose(-1, -2)).view(b, hkv, group, n, m).masked_fill_(~keep[:, None, None], -math.inf)
    p = scores.sub_(scores.amax(dim=-1, keepdim=True)).exp_()
    total = p.sum(dim=-1, keepdim=True)
    out = torch.matmul(p.view(b, hkv, group * n, m), vf).view(b, hkv, group, n, d) / total
    return out.permute(0, 3, 1, 2, 4).reshape(b, n, c["q_heads"], d)[s["seq_of"], s["in_piece"]].to(q.dtype)


def run(s):
    kind = s["case"]["kind"]
    if not own:
        if kind == "chunk":
            return plain_chunk(s, s["q"])
        q, k = plain_rotate(s, s["q"]).to(s["q"].dtype), plain_rotate(s, s["k"])
        if kind == "rope":
            return {"q": q, "k": k.to(s["k"].dtype)}
        k, v = plain_append(s, k, "k"), plain_append(s, s["v"].float(), "v")
        got = {"k": k, "v": v, "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
        return {"q": q, **got} if kind == "append" else {"out": plain_chunk(s, q), **got}
    from paper_2512_19720_b200 import api
    if kind == "rope":
        q, k = api.pd_rope(s["q"], s["k"], s["positions"], s["inv_freq"], axes=s["axes"], interleaved=s["case"]["interleaved"], q_out=s["q_out"], k_out=s["k_out"])
        return {"q": q, "k": k}
    cache = s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"]
    places = s["cu_seqlens"], s["seq_lens"], s["block_table"]
    if kind == "chunk":
        return api.pd_attn_chunk(s["q"], *cache, *places, s["most_new"], s["scale"], out=s["out"])
    # without positions a token has its place in its sequence
    q = api.pd_kv_append_rope(s["q"], s["k"], s["v"], *cache, *places, s["inv_freq"], positions=None if s["axes"] is None else s["positions"], axes=s["axes"],
                              interleaved=s["case"]["interleaved"], q_out=s["q_out"], k_values=s["k_out"], v_values=s["v_out"])
    got = {"k": s["k_out"], "v": s["v_out"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if kind == "append":
        return {"q": q, **got}
    return {"out": api.pd_attn_chunk(q, *cache, *places, s["most_new"], s["scale"], out=s["out"]), **got}


def work(case):
    held, new = lengths(case)
    total = [a + b for a, b in zip(held, new)]
    hq, hkv, d, page, kind = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"], case["kind"]
    n, pairs = sum(new), case["rot"] // 2
    angles = 4 * (pairs + (case["axes"] * n if kind == "rope" or case["axes"] > 1 else 0))
    if kind == "rope":
        return {"bytes": 2 * 2 * n * (hq + hkv) * d + angles, "flops": 6 * n * (hq + hkv) * pairs}
    attended = sum(m * h + m * (m + 1) // 2 for h, m in zip(held, new))
    read = [t if m else 0 for t, m in zip(total, new)]
    chunk = {"bytes": 2 * sum(read) * hkv * d + 8 * hkv * sum(-(-t // page) for t in read) + 2 * 2 * n * hq * d, "flops": 4 * hq * d * attended}
    if kind == "chunk":
        return chunk
    touched = sum(-(-t // page) - h // page for h, t, m in zip(held, total, new) if m)
    again = sum(h % page for h, m in zip(held, new) if m)  # tokens in pages that are gone on with
    # q in and out, k and v in, codes and the values that they stand for out, a scale for each page that is touched, held codes in and out
    append = {"bytes": 2 * 2 * n * hq * d + 2 * n * hkv * d * 5 + 8 * hkv * touched + 2 * 2 * again * hkv * d + angles,
              "flops": 6 * n * (hq + hkv) * pairs + 6 * n * hkv * d}
    if kind == "append":
        return append
    return {"bytes": append["bytes"] + chunk["bytes"], "flops": append["flops"] + chunk["flops"]}


# ---------------------------------------------------------------------------------------------- the definition in 64 bits
def exact_rotation(s, x):
    """A token and pair as a complex number times exp(i t)."""
    c, y, f = s["case"], x.double(), s["inv_freq"].double()
    pairs = len(f)
    p = s["positions"].double()
    t = torch.stack([p[int(s["axes"][i]) if s["axes"] is not None else 0] * f[i] for i in range(pairs)], dim=1)
    first = list(range(0, 2 * pairs, 2)) if c["interleaved"] else list(range(pairs))
    second = [i + 1 for i in first] if c["interleaved"] else [i + pairs for i in first]
    z = torch.complex(y[..., first], y[..., second]) * torch.polar(torch.ones_like(t), t)[:, None]
    y = y.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact_attention(s, q, whole, held, new):
    c, out, at = s["case"], torch.zeros(q.shape, dtype=torch.float64, device="cuda"), 0
    hkv, page = c["kv_heads"], c["page"]
    group = c["q_heads"] // hkv
    for b, (h, n) in enumerate(zip(held, new)):
        if n == 0:
            continue
        pages = s["block_table"][b, :-(-(h + n) // page)].long()
        later = torch.ones(n, h + n, dtype=torch.bool, device="cuda").triu(h + 1)
        for g in range(hkv):
            k, v = (whole[x][pages, g].reshape(-1, c["head_dim"])[:h + n] for x in "kv")
            for i in range(g * group, (g + 1) * group):
                w = torch.softmax((q[at:at + n, i].double() @ k.T * s["scale"]).masked_fill(later, -math.inf), dim=1)
                out[at:at + n, i] = w @ v
        at += n
    return out


def exact(case, seed):
    s = prepare(case, seed)
    held, new = lengths(case)
    page, kind = case["page"], case["kind"]
    if kind == "rope":
        return {"q": exact_rotation(s, s["q"]), "k": exact_rotation(s, s["k"])}
    got, whole = {}, {}
    for name in ("k", "v"):
        codes, scale = s[name + "_codes"].double(), s[name + "_scale"].double()
        if kind != "chunk":
            x, table = exact_rotation(s, s["k"]) if name == "k" else s["v"].double(), s["block_table"].tolist()
            values, at = torch.empty_like(x), 0
            for b, (h, m) in enumerate(zip(held, new)):
                pos = h
                while pos < h + m:  # page by page
                    p, lo = table[b][pos // page], pos % page
                    n = min(page - lo, h + m - pos)
                    y = x[at:at + n].transpose(0, 1)
                    s1 = torch.maximum(y.abs().amax(dim=(1, 2)) / 127, scale[p] if lo else torch.zeros_like(scale[p]))
                    s2 = torch.where(s1 > 0, s1, torch.ones_like(s1))[:, None, None]
                    codes[p, :, :lo] = torch.round(codes[p, :, :lo] * scale[p][:, None, None] / s2)
                    codes[p, :, lo:lo + n] = torch.round(y / s2)
                    scale[p] = s1
                    values[at:at + n] = (codes[p, :, lo:lo + n] * s1[:, None, None]).transpose(0, 1)
                    at, pos = at + n, pos + n
            got[name], got[name + "_scale"] = values, scale
        whole[name] = codes.mul_(scale[:, :, None, None])
    if kind == "chunk":
        return exact_attention(s, s["q"], whole, held, new)
    q = exact_rotation(s, s["q"])
    got = {"k": got["k"], "v": got["v"], "k_scale": got["k_scale"], "v_scale": got["v_scale"]}
    return {"q": q, **got} if kind == "append" else {"out": exact_attention(s, q, whole, held, new), **got}
