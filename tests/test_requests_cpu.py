"""Rotary positions, adapters and log probabilities on the CPU: refusals before any launch, frequencies, the oracle."""
import ctypes
import math

import numpy as np
import pytest

A = pytest.importorskip("paper_2606_12876_amd", reason="libaqmb.so not built")

from oracle import decode  # noqa: E402

S = A.Status
F16, BF16, F32, F8 = 0, 1, 2, 3
NAN, INF = float("nan"), float("inf")


def rotary(**kw):
    a = dict(f=16, rot=32, lay=0, amp=1.0, inv=0, q=16, qs=256, qo=16, qos=256, h=4, k=16, ks=128, ko=16, kos=128, kv=2, dt=BF16,
             dim=64, pos=16, n=3, desc=True)
    a.update(kw)
    d = A.RotaryDesc(a["f"], a["rot"], a["lay"], a["amp"], a["inv"])
    return A.lib.aqmb_rotary(ctypes.byref(d) if a["desc"] else None, a["q"], a["qs"], a["qo"], a["qos"], a["h"], a["k"], a["ks"],
                             a["ko"], a["kos"], a["kv"], a["dt"], a["dim"], a["pos"], a["n"], None)


ROTARY = [
    (dict(desc=False), S.EINVAL), (dict(f=None), S.EINVAL), (dict(f=20), S.EINVAL), (dict(rot=31), S.EINVAL),
    (dict(rot=0), S.EINVAL), (dict(rot=-2), S.EINVAL), (dict(rot=66), S.EINVAL), (dict(lay=2), S.EINVAL), (dict(amp=NAN), S.EINVAL),
    (dict(amp=INF), S.EINVAL), (dict(inv=2), S.EINVAL), (dict(q=None), S.EINVAL), (dict(q=17), S.EINVAL), (dict(qo=None), S.EINVAL),
    (dict(qs=255), S.EINVAL), (dict(qos=255), S.EINVAL), (dict(qs=512), S.EINVAL), (dict(h=0), S.EINVAL),
    (dict(h=65536, qs=1 << 23, qos=1 << 23), S.EUNSUPPORTED),
    (dict(dt=F32), S.EUNSUPPORTED), (dict(dt=F8), S.EUNSUPPORTED), (dict(dim=60), S.EUNSUPPORTED),
    (dict(dim=264, qs=4096, qos=4096), S.EUNSUPPORTED), (dict(pos=None), S.EINVAL), (dict(pos=20), S.EINVAL), (dict(n=0), S.EINVAL),
    (dict(n=1 << 24), S.EUNSUPPORTED), (dict(n=(1 << 23), h=8, qs=512, qos=512), S.EUNSUPPORTED),
]


@pytest.mark.parametrize("kw,status", ROTARY + [
    (dict(k=None), S.EINVAL), (dict(ko=None), S.EINVAL), (dict(kv=0), S.EINVAL), (dict(kv=-1), S.EINVAL), (dict(ks=127), S.EINVAL),
    (dict(kos=127), S.EINVAL), (dict(k=17), S.EINVAL), (dict(ks=256), S.EINVAL), (dict(h=2**31 - 1, kv=2**31 - 1, qs=1 << 40, qos=1 << 40), S.EUNSUPPORTED)])
def test_rotary_refuses(kw, status):
    assert rotary(**kw) == status
    assert A.last_error()


@pytest.mark.parametrize("kw,status", ROTARY + [
    (dict(k=None), S.EINVAL), (dict(v=None), S.EINVAL), (dict(v=17), S.EINVAL), (dict(slots=None), S.EINVAL), (dict(slots=20), S.EINVAL),
    (dict(ks=127), S.EINVAL), (dict(vs=127), S.EINVAL), (dict(cdt=F16), S.EUNSUPPORTED), (dict(cdt=F8), S.EINVAL), (dict(page=0), S.EINVAL)])
def test_rotary_append_refuses(kw, status):
    a = dict(f=16, rot=32, lay=0, amp=1.0, inv=0, q=16, qs=256, qo=16, qos=256, h=4, k=16, ks=128, v=16, vs=128, dt=BF16, dim=64,
             pos=16, n=3, desc=True, cdt=BF16, page=8, slots=16)
    a.update(kw)
    d = A.RotaryDesc(a["f"], a["rot"], a["lay"], a["amp"], a["inv"])
    c = A.KVCacheDesc(16, 16, None, None, 1 << 20, a["cdt"], 0, 4, a["page"], 2, a["dim"])
    assert A.lib.aqmb_rotary_append(ctypes.byref(c), ctypes.byref(d) if a["desc"] else None, a["q"], a["qs"], a["qo"], a["qos"],
                                    a["h"], a["k"], a["ks"], a["v"], a["vs"], a["dt"], a["pos"], a["slots"], a["n"], None) == status
    assert A.last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(desc=False), S.EINVAL), (dict(a=None), S.EINVAL), (dict(b=None), S.EINVAL), (dict(a=17), S.EINVAL), (dict(b=17), S.EINVAL),
    (dict(s=18), S.EINVAL), (dict(r=18), S.EINVAL), (dict(dt=F32), S.EUNSUPPORTED), (dict(dt=F8), S.EUNSUPPORTED), (dict(n=0), S.EINVAL),
    (dict(n=8193), S.EUNSUPPORTED), (dict(rank=0), S.EINVAL), (dict(rank=257), S.EUNSUPPORTED), (dict(din=0), S.EINVAL),
    (dict(dout=0), S.EINVAL), (dict(din=(1 << 23) + 1), S.EUNSUPPORTED), (dict(dout=(1 << 23) + 1), S.EUNSUPPORTED),
    (dict(rows=0), S.EINVAL), (dict(rows=(1 << 22) - 63), S.EUNSUPPORTED),
    (dict(rows=1 << 21, dout=1 << 17, bs=1 << 17, os=1 << 17), S.EUNSUPPORTED),
    (dict(x=None), S.EINVAL), (dict(x=17), S.EINVAL), (dict(xs=99), S.EINVAL), (dict(i=None), S.EINVAL), (dict(i=18), S.EINVAL),
    (dict(base=None), S.EINVAL), (dict(out=None), S.EINVAL), (dict(bs=59), S.EINVAL), (dict(os=59), S.EINVAL),
    (dict(out=16, os=61), S.EINVAL), (dict(out=18, yd=F32), S.EINVAL), (dict(base=17), S.EINVAL), (dict(yd=F8), S.EUNSUPPORTED),
    (dict(ws=None), S.EINVAL), (dict(ws=24), S.EINVAL), (dict(wb=16), S.EINVAL)])
def test_adapters_refuse(kw, status):
    a = dict(a=16, b=16, s=16, r=16, dt=BF16, n=4, rank=8, din=100, dout=60, x=16, xs=100, i=16, rows=5, base=16, bs=60, out=32, os=60,
             yd=BF16, ws=16, wb=1 << 40, desc=True)
    a.update(kw)
    d = A.AdaptersDesc(a["a"], a["b"], a["s"], a["r"], a["dt"], a["n"], a["rank"], a["din"], a["dout"])
    ref = ctypes.byref(d) if a["desc"] else None
    assert A.lib.aqmb_adapters_add(ref, a["x"], a["xs"], a["i"], a["rows"], a["base"], a["bs"], a["out"], a["os"], a["yd"], a["ws"],
                                   a["wb"], None) == status
    assert A.last_error()
    n = ctypes.c_size_t(7)
    if any(k in kw for k in ("a", "b", "s", "r", "dt", "n", "rank", "din", "dout", "rows", "desc")):
        assert A.lib.aqmb_adapters_workspace_bytes(ref, a["rows"], ctypes.byref(n)) == status and n.value == 7
    assert A.lib.aqmb_adapters_workspace_bytes(ref, a["rows"], None) == S.EINVAL


@pytest.mark.parametrize("kw,status", [
    (dict(z=None), S.EINVAL), (dict(z=17), S.EINVAL), (dict(z=18, dt=F32), S.EINVAL), (dict(dt=F8), S.EUNSUPPORTED),
    (dict(st=99), S.EINVAL), (dict(rows=0), S.EINVAL), (dict(rows=(1 << 22) + 1), S.EUNSUPPORTED), (dict(vocab=0), S.EINVAL),
    (dict(scale=0.0), S.EINVAL), (dict(scale=2.0 ** -121), S.EINVAL), (dict(scale=-1.0), S.EINVAL), (dict(scale=NAN), S.EINVAL), (dict(scale=INF), S.EINVAL),
    (dict(t=None), S.EINVAL), (dict(nt=0), S.EINVAL), (dict(nt=-1), S.EINVAL), (dict(lp=None), S.EINVAL), (dict(t=20), S.EINVAL),
    (dict(lp=18), S.EINVAL), (dict(lse=18), S.EINVAL), (dict(ent=18), S.EINVAL), (dict(ids=20), S.EINVAL), (dict(tops=18), S.EINVAL),
    (dict(k=0), S.EINVAL), (dict(ids=None, tops=None), S.EINVAL), (dict(k=-1), S.EINVAL), (dict(k=65), S.EUNSUPPORTED),
    (dict(vocab=4, k=5), S.EINVAL), (dict(t=None, nt=0, lp=None, lse=None, ent=None, ids=None, tops=None, k=0), S.EINVAL),
    (dict(ws=None), S.EINVAL), (dict(wb=100), S.EINVAL), (dict(ws=24), S.EINVAL)])
def test_log_probs_refuse(kw, status):
    a = dict(z=16, dt=BF16, st=100000, rows=2, vocab=100, scale=1.0, t=16, nt=3, lp=16, lse=16, ent=16, ids=16, tops=16, k=5, ws=16,
             wb=1 << 40)
    a.update(vocab=100000 if {"ws", "wb"} & set(kw) else 100)
    a.update(kw)
    assert A.lib.aqmb_log_probs(a["z"], a["dt"], a["st"], a["rows"], a["vocab"], a["scale"], a["t"], a["nt"], a["lp"], a["lse"],
                                a["ent"], a["ids"], a["tops"], a["k"], a["ws"], a["wb"], None) == status
    assert A.last_error()
    n = ctypes.c_size_t(7)
    if any(k in kw for k in ("dt", "rows", "vocab")) or kw.get("k", 5) not in (0, 5):
        assert A.lib.aqmb_log_probs_workspace_bytes(a["dt"], a["rows"], a["vocab"], a["k"], ctypes.byref(n)) == status or "z" in kw
    assert A.lib.aqmb_log_probs_workspace_bytes(a["dt"], 1, 100, 0, None) == S.EINVAL


@pytest.mark.parametrize("kw,status", [
    (dict(dim=7), S.EINVAL), (dict(dim=0), S.EINVAL), (dict(base=1.0), S.EINVAL), (dict(base=NAN), S.EINVAL), (dict(base=INF), S.EINVAL),
    (dict(kind=5), S.EUNSUPPORTED), (dict(kind=-1), S.EUNSUPPORTED), (dict(factor=0.5), S.EINVAL), (dict(factor=NAN), S.EINVAL),
    (dict(kind=3, orig=0), S.EINVAL), (dict(kind=4, low=0.0), S.EINVAL), (dict(kind=3, high=1.0), S.EINVAL), (dict(kind=4, high=NAN), S.EINVAL)])
def test_frequencies_refuse(kw, status):
    a = dict(dim=8, base=10000.0, kind=1, orig=100, factor=2.0, low=1.0, high=4.0)
    a.update(kw)
    out = (ctypes.c_double * 8)(*[-1.0] * 8)
    d = A.RotaryScalingDesc(a["kind"], a["orig"], a["factor"], a["low"], a["high"])
    assert A.lib.aqmb_rotary_frequencies(a["dim"], a["base"], ctypes.byref(d), out, None) == status
    assert list(out) == [-1.0] * 8 and A.last_error()


@pytest.mark.parametrize("dim", [2, 8, 64, 128, 250])
@pytest.mark.parametrize("base,factor,length", [(10000.0, 1.0, 2048), (10000.0, 8.0, 4096), (500000.0, 32.0, 8192), (10.0, 3.0, 7)])
def test_frequencies(dim, base, factor, length):
    """Against the formulas, written as lists; binary64 throughout, a few roundings and a power each (2^-48 is ample)."""
    K = A.RotaryScaling
    plain = [base ** (-2 * i / dim) for i in range(dim // 2)]

    def index(turns):
        return dim * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(base))

    lo, hi = max(math.floor(index(32)), 0), min(math.ceil(index(1)), dim - 1)
    ramp = [min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0) for i in range(dim // 2)]
    turns = [min(max((length / (2 * math.pi / f) - 1) / 3, 0.0), 1.0) for f in plain]
    b2 = base * factor ** (dim / (dim - 2)) if dim > 2 else base
    want = {K.PLAIN: plain, K.LINEAR: [f / factor for f in plain], K.BASE: [b2 ** (-2 * i / dim) for i in range(dim // 2)],
            K.RAMP: [f / factor * t + f * (1 - t) for f, t in zip(plain, ramp)],
            K.TURNS: [f / factor * (1 - t) + f * t for f, t in zip(plain, turns)]}
    for kind, w in want.items():
        f, amp = A.rotary_frequencies(dim, base, kind, factor=factor, original_length=length)
        np.testing.assert_allclose(f.numpy(), w, rtol=2.0 ** -48)
        assert amp == np.float32(0.1 * math.log(factor) + 1 if kind == K.RAMP else 1.0)
    if dim > 2:      # the last one of the larger base is divided by the factor
        assert A.rotary_frequencies(dim, base, K.BASE, factor=factor)[0][-1] == pytest.approx(plain[-1] / factor, rel=1e-12)


def test_the_oracle_itself():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((3, 2, 10))
    ang = rng.standard_normal((3, 4))
    for half in (True, False):
        y = decode.rotary(x, ang, half)
        np.testing.assert_allclose((y ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-12)      # a turn keeps lengths
        np.testing.assert_allclose(decode.rotary(y, -ang, half), x, atol=1e-12)
        assert np.array_equal(y[..., 8:], x[..., 8:])
        # what attention uses: scores depend on the difference of positions
        q, k = rng.standard_normal((2, 1, 1, 10))
        def score(i, j):
            f = np.array([[1.0, 0.3, 0.1, 0.01]])
            return (decode.rotary(q, i * f, half) * decode.rotary(k, j * f, half)).sum()
        assert score(7, 3) == pytest.approx(score(104, 100), abs=1e-10)
    z = rng.standard_normal(9)
    lp, lse, h = decode.log_probs(z)
    assert np.exp(lp).sum() == pytest.approx(1.0) and lse == pytest.approx(np.log(np.exp(z).sum()))
    assert decode.log_probs(np.zeros(8))[2] == pytest.approx(math.log(8))
    assert decode.log_probs(np.array([0.0, -INF]))[2] == 0.0 and h > 0
    a, b = rng.standard_normal((2, 3, 4)), rng.standard_normal((2, 5, 3))
    y = decode.adapted(rng.standard_normal((3, 4)), [1, -1, 2], a, b, np.ones(2), [3, 3])
    assert np.any(y[0]) and not np.any(y[1:])


@pytest.mark.parametrize("scale", [2.36e38, 2.4e38, 3.4028234663852886e38, -3e38])
def test_log_probs_refuse_scales_without_a_finite_factor(scale):
    assert A.lib.aqmb_log_probs(16, BF16, 100, 2, 100, scale, None, 0, None, 16, None, None, None, 0, None, 0, None) == S.EINVAL
    assert "scale" in A.last_error()
