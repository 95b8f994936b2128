"""Norm and rotation, append and attention as a decode step uses them, eagerly, on another stream and from a graph."""
import pytest
import torch

import packed_reference as pr
import window_reference as wr

pytestmark = pytest.mark.gpu
B, H, G, WIDTH = 5, 2, 4, 24
LENS = [0, 15, 16, 100, 371]


@pytest.fixture(scope="module")
def psa():
    import paper_2503_00392_amd as psa
    psa.load_library()
    assert torch.cuda.is_available()
    return psa


class Layer:
    """One layer over a 16-bit cache with a window, one over a 4-bit cache that attends everything."""

    def __init__(self, psa, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()   # noqa: E731
        self.psa = psa
        pages = B * WIDTH
        self.k, self.v = new(pages, H, 16, 128), new(pages, H, 16, 128)
        self.table = torch.randperm(pages, generator=gen, device="cuda").view(B, WIDTH).to(torch.int32)
        self.lens = [torch.tensor(LENS, dtype=torch.int32, device="cuda") for _ in range(2)]
        self.kv = psa.KvCache(self.k, self.v, self.table, self.lens[0], H * G)
        self.meta = psa.build_block_metadata(self.kv)
        self.packed = psa.PackedCache(psa.pack_pages(self.kv, psa.PackedCache.empty_pool(pages, H)), self.table, self.lens[1], H * G, torch.bfloat16)
        self.freq = (10000.0 ** (-torch.arange(0, 128, 2, device="cuda") / 128)).float()
        self.weight = (1 + 0.1 * new(128)).contiguous()
        self.qkv = new(B, (G + 2) * H * 128)
        self.q, self.k_new = torch.empty((B, H * G, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((B, H, 128), dtype=torch.bfloat16, device="cuda")
        self.v_new = torch.empty_like(self.k_new)
        ws = [psa.window_workspace_bytes(self.kv, 50, 4), psa.packed_workspace_bytes(self.packed)]
        self.ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in ws]
        self.out = [torch.empty((B, H * G, 128), device="cuda") for _ in range(2)]
        self.lse = [torch.empty((B, H * G), device="cuda") for _ in range(2)]

    def step(self, stream=None):
        psa, qh = self.psa, H * G * 128
        psa.norm_rotate(self.qkv[:, :qh].view(B, H * G, 128), self.qkv[:, qh:qh + H * 128].view(B, H, 128), self.lens[0], self.freq,
                        q_weight=self.weight, k_weight=self.weight, q_out=self.q, k_out=self.k_new, stream=stream)
        psa.append_kv(self.kv, self.k_new, self.v_new, self.meta, stream=stream)
        psa.append_kv_packed(self.packed, self.k_new, self.v_new, stream=stream)
        psa.window_attention(self.kv, self.q, 50, 4, workspace=self.ws[0], out=self.out[0], lse=self.lse[0], stream=stream)
        psa.packed_attention(self.packed, self.q, workspace=self.ws[1], out=self.out[1], lse=self.lse[1], stream=stream)

    def feed(self, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.qkv.copy_(torch.randn(self.qkv.shape, generator=gen, device="cuda"))
        self.v_new.copy_(torch.randn(self.v_new.shape, generator=gen, device="cuda"))

    def check(self):
        lens, table = self.lens[0].tolist(), self.table.cpu().long()
        assert lens == self.lens[1].tolist()
        for w in self.ws:
            assert self.psa.read_device_error(w) == 0

        def rows(pool):
            return lambda r, at: pool[table[r, at // 16].cuda(), :, (at % 16).cuda()].transpose(0, 1)
        wr.close(self.out[0], self.lse[0], *wr.attention(self.q, rows(self.k), rows(self.v), lens, 50, 4))
        values = [torch.from_numpy(x).cuda() for x in pr.unpack(self.packed.pool.cpu().numpy())]
        wr.close(self.out[1], self.lse[1], *wr.attention(self.q, rows(values[0]), rows(values[1]), lens, 2 ** 31 - 1, 0))


def results(layer):
    return [x.clone() for x in (*layer.out, *layer.lse, layer.q, layer.k_new, layer.packed.pool, *layer.lens)]


def test_a_few_steps(psa):
    layer = Layer(psa, 1)
    for step in range(3):
        layer.feed(step)
        layer.step()
        torch.cuda.synchronize()
        layer.check()
    assert layer.lens[0].tolist() == [n + 3 for n in LENS]


def test_another_stream_and_two_at_once(psa):
    """Two layers' steps on two streams give what one after the other gives."""
    one, two = Layer(psa, 2), Layer(psa, 3)
    for x in (one, two):
        x.feed(9)
        x.step()
    torch.cuda.synchronize()
    want = results(one), results(two)
    one, two = Layer(psa, 2), Layer(psa, 3)
    one.feed(9); two.feed(9)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    one.step(stream=streams[0]); two.step(stream=streams[1])
    torch.cuda.synchronize()
    for layer, w in zip((one, two), want):
        for a, b in zip(results(layer), w):
            assert torch.equal(a, b)


def test_buffers_made_by_the_call_on_another_stream(psa):
    layer = Layer(psa, 4)
    layer.feed(1); layer.step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = []
    for _ in range(4):
        got.append((psa.packed_attention(layer.packed, layer.q, stream=side)[0], psa.window_attention(layer.kv, layer.q, 50, 4, stream=side)[0]))
        torch.randn(1 << 20, device="cuda")                   # the allocator may hand out what the call has let go
    torch.cuda.synchronize()
    for a, b in got:
        assert torch.equal(a, layer.out[1]) and torch.equal(b, layer.out[0])


def test_replays_of_a_captured_step(psa):
    """The step is recorded once; before each replay new inputs and lengths, eager work and synchronizations between them."""
    layer, eager = Layer(psa, 5), Layer(psa, 5)
    layer.feed(0); layer.step()
    eager.feed(0); eager.step()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            layer.step(stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    for step in range(1, 5):
        layer.feed(step); eager.feed(step)
        eager.step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(results(layer), results(eager)):
            assert torch.equal(a, b), step
        layer.check()


def test_two_captured_calls_share_a_workspace(psa):
    """Two graphs over one workspace, replayed in turn on one stream."""
    layer = Layer(psa, 6)
    layer.feed(0); layer.step()
    torch.cuda.synchronize()
    want = [x.clone() for x in layer.out]
    ws = torch.empty(max(x.numel() for x in layer.ws), dtype=torch.uint8, device="cuda")
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graphs[0], stream=side):
            psa.window_attention(layer.kv, layer.q, 50, 4, workspace=ws, out=layer.out[0], lse=layer.lse[0])
        with torch.cuda.graph(graphs[1], stream=side):
            psa.packed_attention(layer.packed, layer.q, workspace=ws, out=layer.out[1], lse=layer.lse[1])
    for _ in range(3):
        for x in layer.out:
            x.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(layer.out[0], want[0]) and torch.equal(layer.out[1], want[1])
