"""Measured cases of the attention operators that stand between the linears of a decoder block: attention over whole
prompts (pd_attn_prompt), writing keys and values into the 8-bit paged cache (pd_kv_append) and attention of single
tokens over that cache (pd_attn_cache).

Head layouts are those of the two block shapes that the library's linears are benchmarked on: 32 query and 32 key/value
heads of 128 (q/k/v 4096 x 4096) and 64 query and 8 key/value heads of 128 (q 8192 x 8192, k/v 1024 x 8192), and small
ones with heads of 64.  Batches (64 decode tokens, 4 prompts of 512 tokens) and prompt lengths (up to 8192 tokens) are
the benchmark's too.

Formulas.  Prompt (token i of a sequence, query head h, key/value head g = h // (q_heads / kv_heads)):
    s[i, j] = scale * q[i, h] . k[j, g]  for j <= i,   out[i, h] = sum_j softmax_j(s[i, :])[j] v[j, g]
Cache: page p, head g holds codes c (int8) and a scale s, and stands for the values c * s.  Appending tokens to a page:
    s' = max(s of what the page holds, max |new values| / 127),  held codes c' = round(c * s / s'),  new codes = round(x / s')
A page whose first token is among the new ones starts from s = 0.  Rounding is to nearest even.
Single tokens: out[b, h] = sum_j softmax_j(scale * q[b, h] . K[j, g]) V[j, g] over the tokens j < seq_lens[b]; an empty sequence
gives zeros.
"""
import math
import random

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
SMALLEST_SCALE = 2.0 ** -120  # a page whose scale is below this holds zeros


def listed():
    def case(name, kind, dtype, q_heads, kv_heads, head_dim, batch, min_len, max_len, lens_seed=1, page=64, held=0, empty=0):
        return {"name": name, "kind": kind, "dtype": dtype, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "batch": batch,
                "min_len": min_len, "max_len": max_len, "lens_seed": lens_seed, "page": page, "held": held, "empty": empty}
    return [
        # a single short prompt through a small layer: what counts is the latency of a call
        case("prompt_short", "prompt", "fp16", 8, 8, 64, 1, 17, 17),
        # the prompts of the multi-variant batch (4 x 512 tokens), 7B heads
        case("prompt_7b_4x512", "prompt", "fp16", 32, 32, 128, 4, 512, 512),
        # a packed batch of prompts of very different lengths, 70B heads
        case("prompt_70b_packed", "prompt", "bf16", 64, 8, 128, 7, 1, 2300, lens_seed=141),
        # one prompt of the longest prefill of the benchmark, 70B heads
        case("prompt_70b_8192", "prompt", "bf16", 64, 8, 128, 1, 8192, 8192),
        # the keys and values of the multi-variant batch's prompts go into fresh pages
        case("append_7b_4x512", "append", "fp16", 32, 32, 128, 4, 512, 512),
        # the next pieces of prompts that are read in pieces: they go on in the middle of a page
        case("append_70b_pieces", "append", "bf16", 64, 8, 128, 9, 1, 1700, lens_seed=3, held=1000),
        # one user, a short conversation, 7B heads: latency again
        case("cache_7b_one", "cache", "fp16", 32, 32, 128, 1, 333, 333),
        # the benchmark's 64 decode tokens, 7B heads, conversations of up to 2112 tokens
        case("cache_7b_64", "cache", "fp16", 32, 32, 128, 64, 100, 2112),
        # 64 decode tokens of which some slots are empty, as in a batch of fixed size, 70B heads, up to 8192 tokens, small pages
        case("cache_70b_64", "cache", "bf16", 64, 8, 128, 64, 200, 8192, page=16, empty=3),
        # two very long conversations: few rows, the work has to be split along the cache
        case("cache_70b_long", "cache", "bf16", 64, 8, 128, 2, 100001, 131072, page=128),
        # a decode step as it is run: each of 64 sequences gets a token and attends over its cache, 70B heads
        case("step_70b_64", "step", "bf16", 64, 8, 128, 64, 1, 2048),
        # a decode step of a small layer with heads of 64
        case("step_small", "step", "fp16", 12, 4, 64, 5, 30, 250, page=32),
    ]


def draw(rng):
    kind = rng.choice(["prompt", "append", "cache", "cache", "step"])
    q_heads, kv_heads = rng.choice([(8, 8), (32, 32), (64, 8), (32, 8), (12, 4), (16, 1), (40, 8), (5, 5)])
    head_dim = rng.choice([64, 128, 128])
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    batch = log(1, 8) if kind in ("prompt", "append") else log(1, 96)
    if kind in ("prompt", "append"):
        most = log(1, 8192 // batch)
    else:
        most = log(1, min(131072, 270_000 * 8 // (batch * kv_heads)))
    least = most if rng.random() < 0.3 else rng.randint(1, most)
    empty = rng.choice([0, 0, 1]) if batch > 2 and kind == "cache" else 0
    return {"kind": kind, "dtype": rng.choice(["fp16", "bf16"]), "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "batch": batch,
            "min_len": least, "max_len": most, "lens_seed": rng.randrange(1000), "page": rng.choice([16, 32, 64, 128]),
            "held": rng.choice([0, 77, 500]) if kind == "append" else 0, "empty": empty}


def lengths(case):
    """(tokens that each sequence holds before the call, tokens of the call): for "cache" all are held, for "step" one is new."""
    r = random.Random(case["lens_seed"])
    lens = [r.randint(case["min_len"], case["max_len"]) for _ in range(case["batch"])]
    for i in r.sample(range(case["batch"]), case["empty"]):
        lens[i] = 0
    if case["kind"] == "cache":
        return lens, [0] * case["batch"]
    if case["kind"] == "step":
        return [n - 1 for n in lens], [1] * case["batch"]
    return [r.randint(0, case["held"]) for _ in lens], lens


def prepare(case, seed):
    dev, dt = torch.device("cuda"), DTYPES[case["dtype"]]
    gen = torch.Generator(device=dev).manual_seed(seed)
    held, new = lengths(case)
    total = [a + b for a, b in zip(held, new)]
    n_new, b, hq, hkv, d = sum(new), case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"]
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=dev, dtype=dt)  # noqa: E731
    # some channels of keys are much larger than others, as they are behind a linear
    channel = 2.0 ** (0.7 * torch.randn(hkv, d, generator=gen, device=dev))
    s = {"case": case, "scale": 1.0 / math.sqrt(d)}
    if case["kind"] in ("prompt", "append", "step"):
        # keys and values of the new tokens are slices of one fused projection's output, as a user's program has them
        qkv = normal(max(n_new, 1), hq + 2 * hkv, d)[:n_new]
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["k"].mul_(channel.to(dt))
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        s["cu_seqlens"] = torch.tensor(cu, dtype=torch.int32, device=dev)
        s["longest"] = max(new)
        s["seq_of"] = torch.repeat_interleave(torch.arange(b, device=dev), torch.tensor(new, device=dev), output_size=n_new)
        s["pos_of"] = torch.arange(n_new, device=dev) - s["cu_seqlens"].long()[s["seq_of"]]
    if case["kind"] == "cache":
        s["q"] = normal(b, hq, d)
    if case["kind"] == "prompt":
        return s
    page = case["page"]
    pages = [-(-n // page) for n in total]
    n_pages = sum(pages) + 8  # a cache has pages that nobody uses
    width = max(max(pages), 1) + 1
    perm = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32)
    at, first = torch.arange(width, device=dev), torch.tensor([sum(pages[:i]) for i in range(b)], device=dev)
    n_of = torch.tensor(pages, device=dev)
    table = torch.where(at[None, :] < n_of[:, None], perm[(first[:, None] + at[None, :]).clamp(max=n_pages - 1)], torch.full((), -1, dtype=torch.int32, device=dev))
    s["block_table"] = table.contiguous()
    s["seq_lens"] = torch.tensor(total, dtype=torch.int32, device=dev)  # with the new tokens
    for name, ch in (("k", channel), ("v", torch.ones_like(channel))):
        codes = torch.empty(n_pages, hkv, page, d, dtype=torch.int8, device=dev)
        scale = torch.empty(n_pages, hkv, dtype=torch.float32, device=dev)
        for i in range(0, n_pages, 4096):  # in pieces: the values in 16 bits need not all be there at once
            x = normal(min(4096, n_pages - i), hkv, page, d) * ch[:, None].to(dt)
            amax = x.abs().amax(dim=(2, 3)).float()
            scale[i:i + 4096] = amax / 127
            codes[i:i + 4096] = torch.round(x.float() * (127 / amax)[:, :, None, None]).to(torch.int8)
        s[name + "_codes"], s[name + "_scale"] = codes, scale
    if case["kind"] in ("append", "step"):
        # for the plain form: the pages that the new tokens touch, the page that each of them goes to, and how many tokens each page holds
        old = torch.tensor(held, device=dev)
        pos = old[s["seq_of"]] + s["pos_of"]
        touched = (at[None, :] >= (old // page)[:, None]) & (at[None, :] < n_of[:, None]) & (torch.tensor(new, device=dev) > 0)[:, None]
        where = touched.nonzero()
        s["touched"] = table[where[:, 0], where[:, 1]].long()
        s["held_in"] = (old[where[:, 0]] - where[:, 1] * page).clamp(min=0, max=page)
        index = torch.zeros(b, width, dtype=torch.long, device=dev)
        index[where[:, 0], where[:, 1]] = torch.arange(len(where), device=dev)
        s["touched_of"] = index[s["seq_of"], pos // page]
        s["slot_of"] = pos % page
        s["k_values"], s["v_values"] = torch.empty(n_new, hkv, d, dtype=dt, device=dev), torch.empty(n_new, hkv, d, dtype=dt, device=dev)
        s["out"] = torch.empty(n_new, hq, d, dtype=dt, device=dev)
    else:
        s["out"] = torch.empty(b, hq, d, dtype=dt, device=dev)
    return s


# ---------------------------------------------------------------------------------------------- the plain forms
def softmax_rows(scores, keep):
    """Softmax over the last axis of the places that `keep` names; zeros where it names none."""
    scores = scores.masked_fill_(~keep, -math.inf)
    top = scores.amax(dim=-1, keepdim=True)
    p = scores.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(dim=-1, keepdim=True)
    return p.div_(torch.where(total == 0, torch.ones_like(total), total))


def plain_prompt(s):
    c, q, k, v = s["case"], s["q"], s["k"], s["v"]
    hkv, d, n = c["kv_heads"], c["head_dim"], s["longest"]
    group = c["q_heads"] // hkv
    cu = s["cu_seqlens"].long()
    at = torch.arange(n, device=q.device)
    inside = at[None, :] < (cu[1:] - cu[:-1])[:, None]
    index = torch.where(inside, cu[:-1, None] + at[None, :], torch.zeros_like(at)[None, :])
    qf = (q.float() * s["scale"])[index].view(-1, n, hkv, group, d).permute(0, 2, 3, 1, 4)
    kf = k.float()[index].permute(0, 2, 1, 3)[:, :, None]
    vf = v.float()[index].permute(0, 2, 1, 3)[:, :, None]
    keep = (at[None, :] <= at[:, None])[None] & inside[:, None, :]
    p = softmax_rows(torch.matmul(qf, kf.transpose(-1, -2)), keep[:, None, None])
    out = torch.matmul(p, vf).permute(0, 3, 1, 2, 4).reshape(-1, n, c["q_heads"], d)
    return out[s["seq_of"], s["pos_of"]].to(q.dtype)


def plain_append_one(s, name):
    x, codes, scale = s[name].float(), s[name + "_codes"], s[name + "_scale"]
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
    return (fresh.float() * after[s["touched_of"]][:, :, None]).to(s[name].dtype)


def plain_cache(s):
    c, q = s["case"], s["q"]
    b, hkv, d, page = c["batch"], c["kv_heads"], c["head_dim"], c["page"]
    group = c["q_heads"] // hkv
    pages = s["block_table"].clamp(min=0).long()
    n = pages.shape[1] * page
    kf = (s["k_codes"][pages].float() * s["k_scale"][pages][..., None, None]).permute(0, 2, 1, 3, 4).reshape(b, hkv, n, d)
    vf = (s["v_codes"][pages].float() * s["v_scale"][pages][..., None, None]).permute(0, 2, 1, 3, 4).reshape(b, hkv, n, d)
    qf = (q.float() * s["scale"]).view(b, hkv, group, d)
    keep = torch.arange(n, device=q.device)[None, :] < s["seq_lens"][:, None]
    p = softmax_rows(torch.matmul(qf, kf.transpose(-1, -2)), keep[:, None, None])
    return torch.matmul(p, vf).view(b, hkv * group, d).to(q.dtype)


def run(s):
    kind = s["case"]["kind"]
    if not own:
        if kind == "prompt":
            return plain_prompt(s)
        if kind == "cache":
            return plain_cache(s)
        k, v = plain_append_one(s, "k"), plain_append_one(s, "v")
        if kind == "append":
            return {"k": k, "v": v, "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
        return {"out": plain_cache(s), "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    from paper_2512_19720_b200 import api
    if kind == "prompt":
        return api.pd_attn_prompt(s["q"], s["k"], s["v"], s["cu_seqlens"], s["scale"])
    cache = s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"]
    if kind == "cache":
        return api.pd_attn_cache(s["q"], *cache, s["seq_lens"], s["block_table"], s["scale"], out=s["out"])
    if kind == "append":
        api.pd_kv_append(s["k"], s["v"], *cache, s["cu_seqlens"], s["seq_lens"], s["block_table"], k_values=s["k_values"], v_values=s["v_values"])
        return {"k": s["k_values"], "v": s["v_values"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    api.pd_kv_append(s["k"], s["v"], *cache, s["cu_seqlens"], s["seq_lens"], s["block_table"])
    out = api.pd_attn_cache(s["q"], *cache, s["seq_lens"], s["block_table"], s["scale"], out=s["out"])
    return {"out": out, "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def work(case):
    held, new = lengths(case)
    total = [a + b for a, b in zip(held, new)]
    hq, hkv, d, page, b = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"], case["batch"]
    n = sum(new)
    touched = sum(-(-t // page) - h // page for h, t, m in zip(held, total, new) if m)
    again = sum(h % page for h, m in zip(held, new) if m)  # tokens in pages that are gone on with
    cache = {"bytes": 2 * sum(total) * hkv * d + 8 * hkv * sum(-(-t // page) for t in total) + 2 * 2 * b * hq * d, "flops": 4 * hq * d * sum(total)}
    if case["kind"] == "prompt":
        return {"bytes": 2 * n * d * (2 * hq + 2 * hkv), "flops": 4 * hq * d * sum(m * (m + 1) // 2 for m in new)}
    if case["kind"] == "cache":
        return cache
    # k and v: 16-bit values in, codes out, a scale for each page that is touched (read too where it held something)
    append = {"bytes": 2 * n * hkv * d * 3 + 8 * hkv * touched + 2 * 2 * again * hkv * d, "flops": 6 * n * hkv * d}
    if case["kind"] == "append":
        return {"bytes": append["bytes"] + 2 * 2 * n * hkv * d, "flops": append["flops"]}  # and the values that the codes stand for
    return {"bytes": append["bytes"] + cache["bytes"], "flops": append["flops"] + cache["flops"]}


# ---------------------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    held, new = lengths(case)
    hkv, d, page = case["kv_heads"], case["head_dim"], case["page"]
    group = case["q_heads"] // hkv
    if case["kind"] == "prompt":
        out, at = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), 0
        for n in new:
            q, k, v = (s[x][at:at + n].double().transpose(0, 1) for x in "qkv")
            later = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
            for h in range(case["q_heads"]):
                w = torch.softmax((q[h] @ k[h // group].T * s["scale"]).masked_fill(later, -math.inf), dim=1)
                out[at:at + n, h] = w @ v[h // group]
            at += n
        return out
    got, whole = {}, {}
    for name in ("k", "v"):
        codes, scale = s[name + "_codes"].double(), s[name + "_scale"].double()
        if case["kind"] != "cache":
            x, table = s[name].double(), s["block_table"].tolist()
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
    if case["kind"] == "append":
        return got
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(a + m for a, m in zip(held, new)):
        if n:
            pages = s["block_table"][b, :-(-n // page)].long()
            k, v = (whole[x][pages].transpose(0, 1).reshape(hkv, -1, d)[:, :n] for x in "kv")
            w = torch.softmax(s["q"][b].double().view(hkv, group, d) @ k.transpose(1, 2) * s["scale"], dim=2)
            out[b] = (w @ v).view(-1, d)
    if case["kind"] == "cache":
        return out
    return {"out": out, "k_scale": got["k_scale"], "v_scale": got["v_scale"]}
