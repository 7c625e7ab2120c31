"""Attention calls inside CUDA graphs: the scratch memory that has to start from zero belongs to one graph."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2512_19720_b200 import api
    return api


class Block:
    """A layer's inputs and cache: prompts, then a token more for each sequence."""

    def __init__(self, api, seed, hq=8, hkv=2, d=128, page=32):
        self.api, lens = api, [700, 1, 2100, 64]
        gen = torch.Generator("cuda").manual_seed(seed)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.x = torch.randn(sum(lens), hq + 2 * hkv, d, generator=gen, device="cuda").half()
        self.y = torch.randn(len(lens), hq + 2 * hkv, d, generator=gen, device="cuda").half()
        self.hq, self.hkv = hq, hkv
        self.cu = i32([0, 700, 701, 2801, 2865])
        self.one = i32([0, 1, 2, 3, 4])
        self.lens, self.longer = i32(lens), i32([n + 1 for n in lens])
        n = [n // page + 1 for n in lens]
        self.table = i32([[sum(n[:b]) + i if i < n[b] else -1 for i in range(max(n))] for b in range(len(n))])
        self.cache = [torch.zeros(sum(n), hkv, page, d, dtype=torch.int8, device="cuda") for _ in range(2)] + [torch.zeros(sum(n), hkv, device="cuda") for _ in range(2)]

    def split(self, x):
        return x[:, :self.hq], x[:, self.hq:self.hq + self.hkv], x[:, self.hq + self.hkv:]

    def run(self, workspace=None):
        q, k, v = self.split(self.x)
        prompt = self.api.pd_attn_prompt(q, k, v, self.cu, workspace=workspace)
        self.api.pd_kv_append(k, v, *self.cache, self.cu, self.lens, self.table, workspace=workspace)
        q, k, v = self.split(self.y)
        self.api.pd_kv_append(k, v, *self.cache, self.one, self.longer, self.table, workspace=workspace)
        return prompt, self.api.pd_attn_cache(q, *self.cache, self.longer, self.table, workspace=workspace)


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_graphs_replayed_in_any_order_and_side_by_side(api):
    blocks = [Block(api, 3 + i) for i in range(3)]
    want = [[t.clone() for t in b.run()] for b in blocks]
    torch.cuda.synchronize()
    graphs, outs, spaces = [], [], []
    for b in blocks:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(b.run())
            spaces.append(api.attn_workspace())
        graphs.append(g)
    spaces.append(api.attn_workspace())
    assert len({t.data_ptr() for t in spaces}) == 4  # none is shared

    def clear():
        for out in outs:
            for t in out:
                t.fill_(float("nan"))
        torch.cuda.synchronize()

    for order in ((2, 1, 0), (1, 2, 0), (0, 0, 2, 1)):
        clear()
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(same(o, w) for o, w in zip(outs, want))
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(5):
        clear()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        eager = blocks[0].api.pd_attn_prompt(*blocks[0].split(blocks[0].x), blocks[0].cu)  # beside them, outside of any graph
        torch.cuda.synchronize()
        assert all(same(o, w) for o, w in zip(outs, want)) and torch.equal(eager, want[0][0])


def test_branches_of_one_graph_have_scratch_of_their_own(api):
    blocks = [Block(api, 13 + i) for i in range(2)]
    want = [[t.clone() for t in b.run()] for b in blocks]
    torch.cuda.synchronize()
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        first, one = blocks[0].run(), api.attn_workspace()
        with torch.cuda.stream(side):
            second, two = blocks[1].run(), api.attn_workspace()
        main.wait_stream(side)
    assert one.data_ptr() != two.data_ptr()
    for _ in range(5):
        for t in (*first, *second):
            t.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert same(first, want[0]) and same(second, want[1])


def test_a_given_workspace_keeps_its_status_over_replays(api):
    block = Block(api, 23)
    ws = torch.zeros(api.workspace_bytes(api.OP_ATTN), dtype=torch.uint8, device="cuda")
    want = [t.clone() for t in block.run(ws)]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = block.run(ws)
    page = block.table[0, 0].clone()
    block.table[0, 0] = -1
    g.replay()
    block.table[0, 0] = page
    g.replay()
    torch.cuda.synchronize()
    assert api.pd_device_status(ws) == 8 and api.pd_device_status(ws) == 0
    g.replay()
    torch.cuda.synchronize()
    assert same(out, want) and api.pd_device_status(ws) == 0
