"""The operators between the layers on other streams than the current one, on two streams at once, and
recorded in a HIP graph that is replayed with other work in between (GPU)."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2606_12876_amd as A  # noqa: E402
from ops_helpers import gen, normal  # noqa: E402

F8 = torch.float8_e4m3fn


def bits(t):
    return t.contiguous().view(torch.uint8)


class Step:
    """A few calls on tensors of their own, the split attention with its workspace among them."""

    def __init__(self, seed, lin):
        g = gen(seed)
        self.lin = lin
        self.h, self.r, self.w = (normal(g, *s, dtype=torch.bfloat16) for s in ((9, 1000), (9, 1000), (1000,)))
        self.r2, self.x8 = torch.zeros_like(self.r), torch.zeros((9, 1000), dtype=torch.int8, device="cuda")
        self.xs, self.y = torch.zeros((9, 16), device="cuda"), torch.zeros((9, 300), device="cuda")
        self.cache = A.KVCache.allocate(40, 16, 2, 64, F8)
        for t in (self.cache.k, self.cache.v):
            bits(t).zero_()
            t.view(torch.uint8).copy_(torch.randint(0, 100, t.shape, generator=g, device="cuda").to(torch.uint8))
        self.cache.k_scale.fill_(0.01)
        self.cache.v_scale.fill_(0.02)
        self.k, self.v = normal(g, 3, 2, 64, dtype=torch.bfloat16), normal(g, 3, 2, 64, dtype=torch.bfloat16)
        self.slots = torch.tensor([5, 100, 639], device="cuda")
        self.src, self.dst = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([3, 4], [20, 21]))
        self.q = normal(g, 2, 8, 64, dtype=torch.bfloat16)
        self.table = torch.full((2, 100), -1, dtype=torch.int32, device="cuda")
        self.table[:, :20] = torch.randperm(40, generator=g, device="cuda").to(torch.int32).view(2, 20)
        self.lens = torch.tensor([320, 77], dtype=torch.int32, device="cuda")
        self.out, self.lse = torch.zeros_like(self.q), torch.zeros((2, 8), device="cuda")

    def run(self, stream=None):
        A.rms_norm(self.h, self.w, self.x8, eps=1e-6, residual=self.r, residual_out=self.r2, scales=self.xs, scale_group=64,
                   stream=stream)
        self.lin.gemv(self.x8, self.y, self.xs, stream=stream)
        A.kv_copy_pages([self.cache], self.src, self.dst, stream=stream)
        self.cache.append(self.k, self.v, self.slots, stream=stream)
        self.cache.attention(self.q, self.table, self.lens, self.out, scale=0.125, lse=self.lse, stream=stream)

    def results(self):
        return [bits(t).clone() for t in (self.r2, self.x8, self.xs, self.y, self.cache.k, self.cache.v, self.cache.k_scale,
                                          self.cache.v_scale, self.out, self.lse)]

    def clear(self):
        for t in (self.r2, self.x8, self.xs, self.y, self.out, self.lse):
            t.zero_()


@pytest.fixture
def layer():
    g = gen(1)
    w = torch.randint(0, 256, (300, 500), generator=g, device="cuda").to(torch.uint8)
    s = (torch.rand((300, 16), generator=g, device="cuda") * 0.01).half()
    lin = A.W4Linear(w, s, group_size=64)
    yield lin
    lin.close()


def expected(seed, layer):
    s = Step(seed, layer)
    assert s.cache.workspace_bytes(8, 2, 1600) > 0         # the attention is split
    s.run()
    torch.cuda.synchronize()
    return s.results()


@pytest.mark.parametrize("raw", [False, True])
def test_a_given_stream(layer, raw):
    """The stream argument, as a torch stream and as a raw handle, while another one is current."""
    want = expected(2, layer)
    s, st = Step(2, layer), torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    big = torch.empty((1 << 26,), device="cuda")
    for rep in range(5):
        with torch.cuda.stream(st):
            big.normal_()                                     # the stream is busy when the calls come
        s.run(stream=st.cuda_stream if raw else st)
        # memory of the workspace must not be handed to other work before the stream is through
        junk = [torch.full((1 << 16,), float("nan"), device="cuda") for _ in range(8)]
        del junk
        st.synchronize()
        for a, b in zip(s.results(), want):
            assert torch.equal(a, b), rep
        s.clear()
        torch.cuda.synchronize()


def test_two_streams_at_once(layer):
    want = [expected(seed, layer) for seed in (2, 3)]
    steps, streams = [Step(2, layer), Step(3, layer)], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                s.run()
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        for a, b in zip(s.results(), w):
            assert torch.equal(a, b)


def test_graph_replays(layer):
    want = expected(4, layer)
    s = Step(4, layer)
    other = torch.randn((1 << 20,), device="cuda")
    s.run()
    torch.cuda.synchronize()
    s.clear()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.run()
    for rep in range(5):
        s.clear()
        other.add_(1.0)                                       # eager work between replays
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(s.results(), want):
            assert torch.equal(a, b), rep
    # the graph reads lengths from the GPU: a longer sequence needs no new recording
    s.lens.copy_(torch.tensor([33, 320], dtype=torch.int32))
    g.replay()
    torch.cuda.synchronize()
    got = s.out.clone()
    s.cache.attention(s.q, s.table, s.lens, s.out, scale=0.125)
    torch.cuda.synchronize()
    assert torch.equal(got, s.out)
    del g


def test_graph_of_the_largest_workgroup():
    """16 heads of 256 on one key-value head: the most LDS the attention takes (over 64 KiB)."""
    g = gen(9)
    c = A.KVCache(normal(g, 64, 1, 8, 256, dtype=torch.bfloat16), normal(g, 64, 1, 8, 256, dtype=torch.bfloat16))
    q = normal(g, 2, 16, 256, dtype=torch.bfloat16)
    table = torch.arange(64, dtype=torch.int32, device="cuda").view(2, 32)
    lens = torch.tensor([256, 100], dtype=torch.int32, device="cuda")
    out, want = torch.empty_like(q), torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.attention(q, table, lens, out, scale=0.06)
    c.attention(q, table, lens, want, scale=0.06)
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    del graph


def test_results_repeat_bit_for_bit(layer):
    s = Step(5, layer)
    s.run()
    first = s.results()
    for _ in range(10):
        s.run()
        for a, b in zip(s.results(), first):
            assert torch.equal(a, b)
