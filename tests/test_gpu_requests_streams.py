"""Rotary positions, adapters and log probabilities on other streams than the current one, on two streams at once, in HIP
graphs replayed with other work in between, and in two graphs that share a workspace (GPU)."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2606_12876_amd as A  # noqa: E402
from ops_helpers import gen, normal  # noqa: E402

BF16 = torch.bfloat16


def bits(t):
    return t.contiguous().view(torch.uint8)


class Step:
    """Every new call once, few rows and many, on tensors of its own."""

    def __init__(self, seed, n):
        g = gen(seed)
        self.n, self.rot = n, A.Rotary.scaled(64)
        self.cache = A.KVCache.allocate(60, 16, 2, 64, torch.float8_e4m3fn)
        for t in (self.cache.k, self.cache.v, self.cache.k_scale, self.cache.v_scale):
            bits(t).zero_()
            t.view(torch.uint8).zero_()
        self.rows, self.pos = normal(g, n, 12, 64, dtype=BF16), torch.randint(0, 9999, (n,), generator=g, device="cuda")
        self.slots = torch.randperm(960, generator=g, device="cuda")[:n]
        self.q, self.q2, self.k2 = (torch.zeros((n, h, 64), dtype=BF16, device="cuda") for h in (8, 8, 2))
        self.ad = A.Adapters(normal(g, 5, 16, 512, dtype=BF16), normal(g, 5, 200, 16, dtype=BF16))
        self.x, self.base = normal(g, n, 512, dtype=BF16), normal(g, n, 200, dtype=BF16)
        self.index = torch.randint(-1, 5, (n,), generator=g, device="cuda").to(torch.int32)
        self.y = torch.zeros_like(self.base)
        self.z, self.t = normal(g, n, 20000, dtype=BF16, std=3.0), torch.randint(0, 20000, (n, 2), generator=g, device="cuda")
        self.lp, self.lse, self.ent = (torch.zeros(s, device="cuda") for s in ((n, 2), (n,), (n,)))
        self.ids, self.tops = torch.zeros((n, 7), dtype=torch.int64, device="cuda"), torch.zeros((n, 7), device="cuda")

    def run(self, stream=None, workspace=None):
        q, k, v = self.rows[:, :8], self.rows[:, 8:10], self.rows[:, 10:]
        self.rot.apply(q, self.pos, self.q2, k=k, k_out=self.k2, inverse=True, stream=stream)
        self.cache.rotary_append(self.rot, q, k, v, self.pos, self.slots, self.q, stream=stream)
        self.ad.add(self.x, self.index, self.base, self.y, workspace=workspace, stream=stream)
        A.log_probs(self.z, self.t, self.lp, lse=self.lse, entropy=self.ent, top_ids=self.ids, top_logprobs=self.tops,
                    workspace=workspace, stream=stream)

    def workspace_bytes(self):
        return max(self.ad.workspace_bytes(self.n), A.log_probs_workspace_bytes(BF16, self.n, 20000, 7))

    def outputs(self):
        return (self.q, self.q2, self.k2, self.y, self.lp, self.lse, self.ent, self.ids, self.tops)

    def results(self):
        c = self.cache
        return [bits(t).clone() for t in self.outputs() + (c.k, c.v, c.k_scale, c.v_scale)]

    def clear(self):
        for t in self.outputs():
            t.zero_()


def equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def expected(seed, n):
    s = Step(seed, n)
    s.run()
    torch.cuda.synchronize()
    return s.results()


SIZES = [3, 250, 300]


@pytest.mark.parametrize("n", SIZES)
@pytest.mark.parametrize("raw", [False, True])
def test_a_given_stream(n, raw):
    want, s, st = expected(1, n), Step(1, n), torch.cuda.Stream()
    torch.cuda.synchronize()
    s.run(stream=st.cuda_stream if raw else st)
    st.synchronize()
    assert equal(s.results(), want)


@pytest.mark.parametrize("n", SIZES)
def test_two_streams_at_once(n):
    want = [expected(i, n) for i in (1, 2)]
    steps, streams = [Step(i, n) for i in (1, 2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                s.run()
    torch.cuda.synchronize()
    assert all(equal(s.results(), w) for s, w in zip(steps, want))


@pytest.mark.parametrize("n", SIZES)
def test_graph_replays(n):
    """One graph, its inputs changed between replays, with eager work and synchronisations between them."""
    other = Step(3, n)
    s = Step(1, n)
    g = torch.cuda.CUDAGraph()
    s.run()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        s.run()
    for seed in (1, 2, 5):
        want, src = expected(seed, n), Step(seed, n)
        for name in ("rows", "pos", "slots", "x", "base", "index", "z", "t"):
            getattr(s, name).copy_(getattr(src, name))
        for t, u in zip((s.ad.a, s.ad.b), (src.ad.a, src.ad.b)):
            t.copy_(u)
        for t in (s.cache.k, s.cache.v, s.cache.k_scale, s.cache.v_scale):
            t.view(torch.uint8).zero_()
        for _ in range(3):
            s.clear()
            g.replay()
            other.run()
            assert float(torch.ones(1000, device="cuda").sum()) == 1000.0
            torch.cuda.synchronize()
            assert equal(s.results(), want)


@pytest.mark.parametrize("n", SIZES)
def test_two_graphs_share_a_workspace(n):
    """In order on one stream, as calls that share one have to be."""
    want, steps = [expected(i, n) for i in (1, 2)], [Step(i, n) for i in (1, 2)]
    ws = torch.empty((max(s.workspace_bytes() for s in steps),), dtype=torch.uint8, device="cuda")
    graphs = []
    for s in steps:
        s.run(workspace=ws)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            s.run(workspace=ws)
    for _ in range(3):
        for s in steps:
            s.clear()
        for g in graphs + graphs[::-1]:
            ws.fill_(255)                              # nothing is kept there from call to call
            g.replay()
        torch.cuda.synchronize()
        assert all(equal(s.results(), w) for s, w in zip(steps, want))


@pytest.mark.parametrize("n", SIZES)
def test_results_repeat_bit_for_bit(n):
    want, s = expected(4, n), Step(4, n)
    for _ in range(10):
        s.clear()
        s.run()
        assert equal(s.results(), want)
