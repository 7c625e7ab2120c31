"""The calls for positions and pieces as they are used: one after another, in CUDA graphs that are replayed in any order, on streams of their own."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2512_19720_b200 import api
    return api


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def offsets(lens):
    return i32([sum(lens[:i]) for i in range(len(lens) + 1)])


class Layer:
    """A layer's queries, keys and values of some sequences, and their empty cache."""

    def __init__(self, api, seed, lens, hq=8, hkv=2, d=128, page=32, dtype=torch.float16):
        self.api, self.lens, self.hq, self.hkv, self.page = api, lens, hq, hkv, page
        gen = torch.Generator("cuda").manual_seed(seed)
        self.x = [torch.randn(n, hq + 2 * hkv, d, generator=gen, device="cuda").to(dtype) for n in lens]
        n = [-(-m // page) for m in lens]
        self.table = i32([[sum(n[:b]) + i if i < n[b] else -1 for i in range(max(n))] for b in range(len(n))])
        self.inv_freq = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).float().cuda()
        self.shape = (sum(n), hkv, page, d)
        self.clear()

    def clear(self):
        self.cache = [torch.zeros(self.shape, dtype=torch.int8, device="cuda") for _ in range(2)] + [torch.zeros(self.shape[:2], device="cuda") for _ in range(2)]

    def split(self, x):
        return x[:, :self.hq], x[:, self.hq:self.hq + self.hkv], x[:, self.hq + self.hkv:]

    def piece(self, held, new, most=0, workspace=None, chunk_workspace=None):
        """The next `new` tokens of each sequence; returns their outputs."""
        q, k, v = self.split(torch.cat([x[h:h + n] for x, h, n in zip(self.x, held, new)]))
        places = offsets(new), i32([h + n for h, n in zip(held, new)]), self.table
        q = self.api.pd_kv_append_rope(q, k, v, *self.cache, *places, self.inv_freq, workspace=workspace)
        return self.api.pd_attn_chunk(q, *self.cache, *places, most, workspace=chunk_workspace)


def relative(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64)])
def test_pieces_agree_with_whole_prompts(api, hq, hkv, d, dtype):
    """Sequences read in pieces of any sizes, single tokens among them, against pd_rope and pd_attn_prompt on the whole, which keep keys and values
    in 16 bits.  A code is off by half a step of amax / 127 at most: about 0.9 % of a normal value's deviation (amax of a page's thousands of
    values is near 4 deviations: 4 / 127 / sqrt(12)); weights of averages over independent tokens scale signal and error alike, scores move by
    the same fraction of their deviation; 3 % leaves room for both, and for codes that are rounded again as a page's scale grows."""
    lens = [300, 1, 517]
    layer = Layer(api, 3, lens, hq, hkv, d, dtype=dtype)
    whole = torch.cat(layer.x)
    q, k, v = layer.split(whole)
    positions = torch.cat([torch.arange(n, device="cuda") for n in lens]).int()
    q, k = api.pd_rope(q, k, positions, layer.inv_freq)
    want = api.pd_attn_prompt(q, k, v, offsets(lens)).split(lens)
    held, got = [0, 0, 0], [[], [], []]
    for new in ([200, 1, 3], [1, 0, 1], [0, 0, 500], [99, 0, 13]):
        out = layer.piece(held, new, most=max(new)).split(new)
        for b, n in enumerate(new):
            got[b].append(out[b])
            held[b] += n
    assert held == lens
    for b in range(3):
        assert relative(torch.cat(got[b]), want[b]) < 0.03
    assert api.pd_device_status(api.attn_workspace()) == 0 and api.pd_device_status(api.chunk_workspace()) == 0


def steps(layer, workspace=None, chunk_workspace=None):
    layer.clear()
    held, outs = [0] * len(layer.lens), []
    for new in ([n - 40 for n in layer.lens], [36] * len(layer.lens), [3] * len(layer.lens), [1] * len(layer.lens)):
        outs.append(layer.piece(held, new, max(new), workspace, chunk_workspace))
        held = [h + n for h, n in zip(held, new)]
    return outs


def test_graphs_replayed_in_any_order_and_side_by_side(api):
    layers = [Layer(api, 5 + i, [700, 64, 2100]) for i in range(3)]
    want = [[t.clone() for t in steps(layer)] for layer in layers]
    torch.cuda.synchronize()
    graphs, outs, spaces = [], [], []
    pieces = [[(layer.split(torch.cat([x[h:h + n] for x, h, n in zip(layer.x, held, new)])), offsets(new), i32([h + n for h, n in zip(held, new)]), max(new))
               for held, new in (([0] * 3, [n - 40 for n in layer.lens]), ([n - 40 for n in layer.lens], [36] * 3), ([n - 4 for n in layer.lens], [3] * 3),
                                 ([n - 1 for n in layer.lens], [1] * 3))] for layer in layers]
    torch.cuda.synchronize()
    for layer, todo in zip(layers, pieces):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = []
            for (q, k, v), cu, lens, most in todo:
                q = api.pd_kv_append_rope(q, k, v, *layer.cache, cu, lens, layer.table, layer.inv_freq)
                got.append(api.pd_attn_chunk(q, *layer.cache, cu, lens, layer.table, most))
            outs.append(got)
            spaces.append(api.chunk_workspace())
        graphs.append(g)
    spaces.append(api.chunk_workspace())
    assert len({t.data_ptr() for t in spaces}) == 4  # none is shared
    streams = [torch.cuda.Stream() for _ in graphs]
    for order in ([0, 1, 2], [2, 0, 1, 1, 2, 0]):
        for i in order:
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        torch.cuda.synchronize()
        for got, w in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(got, w))


def test_streams_of_their_own(api):
    layers = [Layer(api, 11 + i, [400, 90]) for i in range(3)]
    want = [[t.clone() for t in steps(layer)] for layer in layers]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in layers], [None] * 3
    for _ in range(3):
        for i, (layer, s) in enumerate(zip(layers, streams)):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got[i] = steps(layer)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


def test_given_workspaces_and_many_calls_on_one(api):
    layer = Layer(api, 17, [200, 50])
    want = [t.clone() for t in steps(layer)]
    one, two = (torch.zeros(api.workspace_bytes(op), dtype=torch.uint8, device="cuda") for op in (api.OP_ATTN, api.OP_ATTN_CHUNK))
    two[1 << 17:] = 255  # what need not be zero
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(steps(layer, one, two), want))
    assert api.pd_device_status(one) == 0 and api.pd_device_status(two) == 0
    # a call that reports leaves the workspace as the next one needs it
    q = layer.split(layer.x[0][:1])[0]
    api.pd_attn_chunk(q, *layer.cache, offsets([1, 0]), i32([10 ** 6, 5]), layer.table, 1, workspace=two)
    assert api.pd_device_status(two) == 8 and api.pd_device_status(two) == 0
    assert all(torch.equal(a, b) for a, b in zip(steps(layer, one, two), want))


def test_binding_refusals(api):
    layer = Layer(api, 19, [64])
    q, k, v = layer.split(layer.x[0])
    cu, lens = offsets([64]), i32([64])
    p = torch.arange(64, device="cuda", dtype=torch.int32)
    for bad in (dict(positions=p[:-1]), dict(positions=p.long()), dict(positions=p.cpu()), dict(axes=p[:5]), dict(inv_freq=layer.inv_freq.double()), dict(q_out=q[:1]),
                dict(positions=None), dict(k=k[:3]), dict(positions=p.float())):
        args = dict(q=q, k=k, positions=p, inv_freq=layer.inv_freq)
        args.update(bad)
        with pytest.raises((TypeError, ValueError)):
            api.pd_rope(**args)
    with pytest.raises(api.PdError):
        api.pd_rope(q, k, p, layer.inv_freq[:12])
    with pytest.raises(api.PdError):
        api.pd_rope(q, k, torch.stack([p, p]), layer.inv_freq)  # two axes and no word on which pair turns with which
    with pytest.raises((TypeError, ValueError)):
        api.pd_kv_append_rope(q[:5], k, v, *layer.cache, cu, lens, layer.table, layer.inv_freq)
    with pytest.raises((TypeError, ValueError)):
        api.pd_attn_chunk(q, *layer.cache, cu.long(), lens, layer.table)
    with pytest.raises((TypeError, ValueError)):
        api.pd_attn_chunk(q.float(), *layer.cache, cu, lens, layer.table)
    with pytest.raises(api.PdError):
        api.pd_attn_chunk(q, *layer.cache, cu, lens, layer.table, max_new=-3)
