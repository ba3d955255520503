"""Rotary positions, adapters and log probabilities past ctypes: taken for the usual arguments, with the results of the other
way, and left alone for all else."""
import pytest
import torch

A = pytest.importorskip("paper_2606_12876_amd", reason="libaqmb.so not built")
from paper_2606_12876_amd import _direct  # noqa: E402

FUNCTIONS = ("rotary", "rotary_append", "adapters_add", "log_probs")


def test_leaves_what_it_does_not_know():
    for n in (0, 1, 7, 9, 10):
        for name in FUNCTIONS:
            for bad in (None, 1, "x", [], torch.zeros(2, 3), torch.zeros(0), torch.zeros(2, 8, dtype=torch.float16)):
                assert getattr(_direct, name)(*([bad] * n)) is None
    with pytest.raises(TypeError):
        _direct.bind_requests(1, 2)
    with pytest.raises(ValueError):
        _direct.bind_requests(0, 0, 0, 0, 0, 0)


def normal(*shape, dtype=torch.bfloat16):
    return torch.randn(*shape, device="cuda").to(dtype)


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


class Counted:
    """_direct with its answers noted."""

    def __init__(self):
        self.seen = []

    def __getattr__(self, name):
        def call(*a):
            r = getattr(_direct, name)(*a)
            self.seen.append((name, r))
            return r
        return call


@pytest.fixture
def counted(monkeypatch):
    c = Counted()
    monkeypatch.setattr(A, "_direct", c)
    return c


def both(counted, monkeypatch, call, outs):
    """call() past ctypes and through it: the former is taken, the results are the same."""
    got = []
    for direct in (counted, None):
        monkeypatch.setattr(A, "_direct", direct)
        for t in outs:
            t.view(torch.uint8).zero_() if t.is_contiguous() else t.zero_()
        call()
        got.append([t.clone() for t in outs])
    monkeypatch.setattr(A, "_direct", counted)
    assert counted.seen[-1][1] == 0
    assert all(same(a, b) for a, b in zip(*got))


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 5])
def test_the_same_results(counted, monkeypatch, n):
    r = A.Rotary.scaled(64, layout="interleaved")
    rows = normal(n, 10, 64)
    q, k, v, pos = rows[:, :6], rows[:, 6:8], rows[:, 8:], torch.arange(n, device="cuda") * 1000
    qo, ko = normal(2 * n, 6, 64)[::2], normal(n, 2, 64)
    for inverse in (False, True):
        both(counted, monkeypatch, lambda: r.apply(q, pos, qo, k=k, k_out=ko, inverse=inverse), [qo, ko])
    both(counted, monkeypatch, lambda: r.apply(q, pos, qo), [qo])
    c = A.KVCache.allocate(4, 8, 2, 64, torch.float8_e4m3fn)
    slots = torch.randperm(32, device="cuda")[:n]
    both(counted, monkeypatch, lambda: c.rotary_append(r, q, k, v, pos, slots, qo), [qo, c.k, c.v, c.k_scale, c.v_scale])
    ad = A.Adapters(normal(3, 16, 80), normal(3, 48, 16), torch.rand(3, device="cuda"))
    x, idx, base, out = normal(n, 96)[:, :80], torch.arange(n, device="cuda").to(torch.int32) % 4 - 1, normal(n, 48), normal(n, 50)[:, :48]
    both(counted, monkeypatch, lambda: ad.add(x, idx, base, out), [out])
    ws = torch.empty(ad.workspace_bytes(n), dtype=torch.uint8, device="cuda")
    both(counted, monkeypatch, lambda: ad.add(x, idx, base, out, workspace=ws), [out])
    z, t = normal(n, 9000, dtype=torch.float32), torch.arange(n, device="cuda")
    lp, lse, ent, ids, tops = (torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"),
                               torch.zeros(n, 4, dtype=torch.int64, device="cuda"), torch.zeros(n, 4, device="cuda"))
    both(counted, monkeypatch, lambda: A.log_probs(z, t, lp, scale=0.5, lse=lse, entropy=ent, top_ids=ids, top_logprobs=tops),
         [lp, lse, ent, ids, tops])
    both(counted, monkeypatch, lambda: A.log_probs(z, top_ids=ids[:, :1].contiguous(), lse=lse), [lse])


@pytest.mark.gpu
def test_left_alone(counted):
    """What the module does not take comes back None and is refused, or taken, by the binding."""
    r, q, pos = A.Rotary.scaled(64), normal(2, 3, 64), torch.zeros(2, dtype=torch.int64, device="cuda")
    ad, x = A.Adapters(normal(1, 8, 64), normal(1, 32, 8)), normal(2, 64)
    i, b = torch.zeros(2, dtype=torch.int32, device="cuda"), normal(2, 32)
    z, f = normal(2, 30), torch.zeros(2, device="cuda")
    for call in (lambda: r.apply(q, pos.int(), q), lambda: r.apply(q.cpu(), pos, q), lambda: r.apply(q, pos, q.float()),
                 lambda: r.apply(q, pos, q, k=q), lambda: r.apply(q.transpose(0, 1), pos, q), lambda: ad.add(x.half(), i, b, b),
                 lambda: ad.add(x, i.long(), b, b), lambda: ad.add(x, i, b, b[:1]), lambda: A.log_probs(z, lse=f[:1]),
                 lambda: A.log_probs(z, i.long()), lambda: A.log_probs(z[0], lse=f)):
        with pytest.raises(A.AqmbError):
            call()
        assert counted.seen[-1][1] is None
    # the library's own refusals come back as its status
    with pytest.raises(A.AqmbError, match="scale"):
        A.log_probs(z, lse=f, scale=-1.0)
    assert counted.seen[-1][1] == A.Status.EINVAL
    with pytest.raises(A.AqmbError, match="output"):
        A.log_probs(z)
    A.log_probs(z, lse=f, scale=2)                     # an integer: by ctypes
    assert counted.seen[-1][1] is None


@pytest.mark.gpu
def test_the_current_stream(counted):
    r, q, pos = A.Rotary.scaled(64), normal(2000, 8, 64), torch.arange(2000, device="cuda")
    want, out = torch.empty_like(q), torch.zeros_like(q)
    r.apply(q, pos, want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        r.apply(q, pos, out)
    assert counted.seen[-1][1] == 0
    s.synchronize()
    assert torch.equal(out, want)
