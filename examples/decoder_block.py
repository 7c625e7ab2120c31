"""The attention half of a decoder block served from a packed delta: prompts, then tokens one at a time.

    x -> q, k, v = pd_linear(x, W_b of q/k/v, delta) -> attention -> y = pd_linear(., W_b of o, delta)

Prompts of several sequences are packed into one batch: pd_attn_prompt attends inside each of them and pd_kv_append writes
their keys and values into the 8-bit cache.  Every further token of a sequence is a row of a decode batch: pd_kv_append adds
it to its page and pd_attn_cache attends over the cache.  Norms, positions and the MLP half are left out.

    python examples/decoder_block.py [--q-heads 32 --kv-heads 8 --head-dim 128 --steps 16]

prints how far the tokens decoded one by one are from the same tokens as part of longer prompts, which keep keys and values in
16 bits: what the 8-bit cache costs.  Weights are synthetic.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2512_19720_b200 import api, synth_torch  # noqa: E402


class DeltaLinear:
    """A linear layer of a fine-tuned model: the shared base weights, a sign mask and scales."""

    def __init__(self, d_out, d_in, seed, device):
        self.w_b = synth_torch.gen_base(d_out, d_in, seed, device)
        w_f = synth_torch.gen_finetuned(self.w_b, seed + 1000)
        self.mask, self.v, _ = api.pd_pack_delta(w_f, self.w_b, want_col=False)

    def __call__(self, x):
        return api.pd_linear(x, self.w_b, self.mask, self.v, api.AXIS_ROW, weights_resident=True)


class AttentionBlock:
    def __init__(self, q_heads, kv_heads, head_dim, n_seqs, max_tokens, page=64, seed=0, device="cuda"):
        self.q_heads, self.kv_heads, self.head_dim, self.page = q_heads, kv_heads, head_dim, page
        width = q_heads * head_dim
        # one base matrix for q, k and v: the three are slices of its output, which the attention calls take as they are
        self.qkv = DeltaLinear((q_heads + 2 * kv_heads) * head_dim, width, seed, device)
        self.o = DeltaLinear(width, width, seed + 1, device)
        pages_per_seq = -(-max_tokens // page)
        shape = (n_seqs * pages_per_seq, kv_heads, page, head_dim)
        self.k_codes, self.v_codes = (torch.zeros(shape, dtype=torch.int8, device=device) for _ in range(2))
        self.k_scale, self.v_scale = (torch.zeros(shape[:2], dtype=torch.float32, device=device) for _ in range(2))
        # this example gives every sequence its pages at once, in any order; a server would hand them out as they are needed
        order = torch.randperm(shape[0], generator=torch.Generator().manual_seed(seed)).to(torch.int32)
        self.block_table = order.view(n_seqs, pages_per_seq).to(device)
        self.seq_lens = torch.zeros(n_seqs, dtype=torch.int32, device=device)
        self.one_each = torch.arange(n_seqs + 1, dtype=torch.int32, device=device)

    def project(self, x):
        qkv = self.qkv(x).view(x.shape[0], -1, self.head_dim)
        return qkv[:, :self.q_heads], qkv[:, self.q_heads:self.q_heads + self.kv_heads], qkv[:, self.q_heads + self.kv_heads:]

    def cache(self):
        return self.k_codes, self.v_codes, self.k_scale, self.v_scale

    def prompt(self, x, cu_seqlens, keep=True):
        """x [T, width], the sequences' tokens one after another; with keep their keys and values go into the (empty) cache."""
        q, k, v = self.project(x)
        out = api.pd_attn_prompt(q, k, v, cu_seqlens)
        if keep:
            self.seq_lens.copy_(cu_seqlens[1:] - cu_seqlens[:-1])
            api.pd_kv_append(k, v, *self.cache(), cu_seqlens, self.seq_lens, self.block_table)
        return self.o(out.view(x.shape[0], -1))

    def step(self, x):
        """x [n_seqs, width]: the next token of every sequence."""
        q, k, v = self.project(x)
        self.seq_lens += 1
        api.pd_kv_append(k, v, *self.cache(), self.one_each, self.seq_lens, self.block_table)
        return self.o(api.pd_attn_cache(q, *self.cache(), self.seq_lens, self.block_table).view(x.shape[0], -1))


def offsets(lens, device):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=device)


def run(q_heads=32, kv_heads=8, head_dim=128, lens=(300, 17, 1000, 64), steps=16, device="cuda"):
    """Relative difference (2-norm) of the tokens decoded one by one from the same tokens in longer prompts."""
    block = AttentionBlock(q_heads, kv_heads, head_dim, len(lens), max(lens) + steps, device=device)
    gen = torch.Generator(device).manual_seed(7)
    tokens = [torch.randn(n + steps, q_heads * head_dim, generator=gen, device=device).half() for n in lens]
    block.prompt(torch.cat([t[:n] for t, n in zip(tokens, lens)]), offsets(lens, device))
    stepped = [block.step(torch.stack([t[n + i] for t, n in zip(tokens, lens)])) for i in range(steps)]
    longer = [n + steps for n in lens]
    whole = block.prompt(torch.cat(tokens), offsets(longer, device), keep=False)
    assert api.pd_device_status(api.attn_workspace()) == 0 and api.pd_device_status() == 0
    ends = offsets(longer, device).tolist()[1:]
    want = torch.stack([torch.stack([whole[e - steps + i] for e in ends]) for i in range(steps)]).double()
    got = torch.stack(stepped).double()
    return float((got - want).norm() / want.norm())


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--q-heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--head-dim", type=int, default=128)
    ap.add_argument("--steps", type=int, default=16)
    a = ap.parse_args()
    off = run(a.q_heads, a.kv_heads, a.head_dim, steps=a.steps)
    print(f"{a.steps} tokens of 4 sequences decoded over the 8-bit cache: {off:.2e} from the same tokens in prompts (relative, 2-norm)")


if __name__ == "__main__":
    main()
