"""Rotary positions, alone and into a paged cache, against the oracle in 64 bits (GPU).

Tolerance of a turned value a c - b s of output type T, with v = amplitude (|a| + |b|): sine and cosine are off by at most 2^-22 (times
the amplitude), and by the angle's own error: two binary64 roundings of position * frequency here, one in the oracle, 3 * 2^-53 |angle|
together; the two products and the sum round by u = 2^-24 each; then half a step of T at the exact value, whose step
may be the next one up after these errors: v (2^-22 + 2^-51 |angle| + 4 u), and half an ulp of |exact| + that."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import decode

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2606_12876_amd as A  # noqa: E402
from ops_helpers import U, gen, half_ulp, normal, values  # noqa: E402

F8 = torch.float8_e4m3fn
LAYOUTS = ["half", "interleaved"]


def angles_of(rot, positions):
    return np.outer(positions.cpu().numpy().astype(np.float64), rot.frequencies.cpu().numpy())


def partner(x, pairs, half):
    """|a| + |b| of every value's pair, 0 behind the pairs."""
    v = np.zeros_like(x)
    for i in range(pairs):
        a, b = (i, i + pairs) if half else (2 * i, 2 * i + 1)
        v[..., a] = v[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return v


def bound(x, ang, rot):
    """What the turned value may be off before its rounding."""
    pairs = ang.shape[1]
    far = np.zeros((x.shape[0], 1, x.shape[2]))
    for i in range(pairs):
        a, b = (i, i + pairs) if rot.layout == "half" else (2 * i, 2 * i + 1)
        far[:, 0, a] = far[:, 0, b] = np.abs(ang[:, i])
    return abs(rot.amplitude) * partner(x, pairs, rot.layout == "half") * (2.0 ** -22 + 4 * U + 2.0 ** -51 * far)


def check(got, x, ang, rot, dtype, inverse=False):
    want = decode.rotary(x, -ang if inverse else ang, rot.layout == "half", rot.amplitude)
    e = bound(x, ang, rot)
    assert np.all(np.abs(values(got) - want) <= e + half_ulp(np.abs(want) + e, dtype))
    d = 2 * ang.shape[1]
    assert np.array_equal(values(got)[..., d:], x[..., d:])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("n,heads,kv,dim,rot", [(1, 1, 1, 8, 2), (1, 32, 8, 128, 128), (3, 5, 2, 64, 32), (2, 7, 7, 80, 58), (5, 3, 1, 256, 256),
                                                (33, 40, 20, 96, 48), (130, 9, 3, 200, 22), (4, 17, 1, 128, 96), (700, 6, 2, 64, 64)])
def test_rotary(n, heads, kv, dim, rot, layout, dtype):
    g = gen(n + dim + rot)
    r = A.Rotary.scaled(rot, layout=layout, scaling=A.RotaryScaling.RAMP, factor=4.0, original_length=512)
    rows = normal(g, n, heads + 2 * kv, dim, dtype=dtype)                       # a fused projection's rows
    q, k = rows[:, :heads], rows[:, heads:heads + kv]
    pos = torch.randint(0, 100000, (n,), generator=g, device="cuda")
    pos[0] = 0
    for inverse in (False, True):
        qo, ko = torch.empty((n * 2, heads, dim), dtype=dtype, device="cuda")[::2], torch.empty((n, kv, dim), dtype=dtype, device="cuda")
        r.apply(q, pos, qo, k=k, k_out=ko, inverse=inverse)
        ang = angles_of(r, pos)
        check(qo, values(q), ang, r, dtype, inverse)
        check(ko, values(k), ang, r, dtype, inverse)
    # queries alone, and in place
    q1 = torch.empty_like(qo)
    A.rotary(r, q, pos, q1, inverse=True)
    assert torch.equal(q1, qo)
    v = rows[:, heads + kv:].clone()
    r.apply(q, pos, q, k=k, k_out=k, inverse=True)
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(rows[:, heads + kv:], v)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_far_negative_and_odd_positions(layout):
    g = gen(5)
    r = A.Rotary.scaled(128, layout=layout)
    pos = torch.tensor([0, 1, -1, 131071, 2 ** 27, -2 ** 31, 2 ** 33 + 1, 10 ** 6], device="cuda")
    q = normal(g, len(pos), 4, 128, dtype=torch.float16)
    out = torch.empty_like(q)
    r.apply(q, pos, out)
    assert torch.equal(out[0], q[0])
    check(out, values(q), angles_of(r, pos), r, torch.float16)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_infinities_and_nan_stay_in_their_pairs(layout):
    g = gen(6)
    r = A.Rotary.scaled(48, layout=layout)
    q = normal(g, 2, 3, 80, dtype=torch.bfloat16)
    q[0, 1, 3], q[1, 2, 60], q[0, 0, 79] = float("nan"), float("inf"), -float("inf")
    out = torch.empty_like(q)
    r.apply(q, torch.tensor([5, 9], device="cuda"), out)
    a, b = (3, 27) if layout == "half" else (2, 3)
    bad = torch.zeros_like(q, dtype=torch.bool)
    bad[0, 1, a] = bad[0, 1, b] = bad[1, 2, 60] = bad[0, 0, 79] = True
    assert torch.equal(out.isfinite(), ~bad)
    assert out[1, 2, 60] == float("inf") and out[0, 0, 79] == -float("inf")


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("rot,dim", [(64, 64), (20, 48)])
def test_the_inverse_is_the_gradient(layout, rot, dim):
    """d/dq of <w, turn(q)> is w turned back: against autograd of the formula, and against differences of the formula,
    which is linear, so differences of any width are exact but for binary64's roundings."""
    g = gen(7)
    r = A.Rotary.scaled(rot, layout=layout, scaling=A.RotaryScaling.RAMP, factor=2.0, original_length=64)
    pos = torch.randint(0, 5000, (6,), generator=g, device="cuda")
    w = normal(g, 6, 3, dim, dtype=torch.float16)
    grad = torch.empty_like(w)
    r.apply(w, pos, grad, inverse=True)
    ang = angles_of(r, pos)
    x, ww = np.random.default_rng(0).standard_normal((6, 3, dim)), values(w)
    f = lambda v: (decode.rotary(v, ang, layout == "half", r.amplitude) * ww).sum()  # noqa: E731
    e = bound(ww, ang, r)
    for t, h, i in [(0, 0, 0), (3, 2, 5), (5, 1, rot - 1), (2, 0, rot // 2), (1, 1, dim - 1)]:
        d = np.zeros_like(x)
        d[t, h, i] = 1.0
        want = (f(x + d) - f(x - d)) / 2
        assert abs(values(grad)[t, h, i] - want) <= e[t, h, i] + half_ulp(np.abs(want) + e[t, h, i], torch.float16) + 1e-10
    leaf = torch.tensor(x, requires_grad=True)
    c, s = torch.tensor(np.cos(ang))[:, None], torch.tensor(np.sin(ang))[:, None]
    p = rot // 2
    a, b = (leaf[..., :p], leaf[..., p:rot]) if layout == "half" else (leaf[..., 0:rot:2], leaf[..., 1:rot:2])
    wt = torch.tensor(ww)
    wa, wb = (wt[..., :p], wt[..., p:rot]) if layout == "half" else (wt[..., 0:rot:2], wt[..., 1:rot:2])
    (r.amplitude * ((a * c - b * s) * wa + (b * c + a * s) * wb).sum() + (leaf[..., rot:] * wt[..., rot:]).sum()).backward()
    want = leaf.grad.numpy()
    assert np.all(np.abs(values(grad) - want) <= e + half_ulp(np.abs(want) + e, torch.float16) + 1e-12)


def bits(t):
    return t.contiguous().view(torch.uint8)


def filled(g, pages, page, kv, dim, dtype, layout):
    c = A.KVCache.allocate(pages, page, kv, dim, dtype, layout=layout)
    for t in (c.k, c.v):
        bits(t).copy_(torch.randint(0, 120, bits(t).shape, generator=g, device="cuda").to(torch.uint8))
    for t in (c.k_scale, c.v_scale):
        if t is not None:
            t.uniform_(0.5, 1.5, generator=g)
    return c


def copy_of(c):
    return A.KVCache(*(None if t is None else t.clone() for t in (c.k, c.v, c.k_scale, c.v_scale)), layout=c.layout)


def by_slot(c, t):
    t = t.transpose(1, 2) if c.layout == "head" else t
    return t.reshape(c.n_pages * c.page_size, c.n_kv_heads, *t.shape[3:])


@pytest.mark.parametrize("cache,dtype", [(torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16), (F8, torch.float16),
                                         (F8, torch.bfloat16)])
@pytest.mark.parametrize("order", ["head", "slot"])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("n,pages,page,heads,kv,dim,rot", [(1, 3, 16, 2, 2, 64, 64), (5, 6, 1, 1, 1, 8, 6), (37, 9, 7, 9, 3, 80, 32), (64, 5, 20, 32, 8, 128, 128),
                                                           (20, 3, 8, 5, 5, 256, 100), (300, 20, 16, 4, 1, 200, 200)])
def test_rotary_append(n, pages, page, heads, kv, dim, rot, layout, order, cache, dtype):
    """16 bits: the two calls' results, to the bit. 8 bits: keys by the scaling of the exact turned values, whose
    largest is off by their bound e: scales within (4 u + e / largest) of themselves, values by half a step of the grid and
    what that and e change of it; values v to the bit as append writes them."""
    g = gen(n + dim)
    c = filled(g, pages, page, kv, dim, cache, order)
    r = A.Rotary.scaled(rot, layout=layout)
    rows = normal(g, n, heads + 2 * kv, dim, dtype=dtype)
    q, k, v = rows[:, :heads], rows[:, heads:heads + kv], rows[:, heads + kv:]
    v[0, 0] = 0.0
    pos = torch.randint(0, 9000, (n,), generator=g, device="cuda")
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:n].clone()
    if n > 2:
        slots[1], slots[2] = -1, pages * page
    two = copy_of(c)
    qo, q2, k2 = torch.empty((n, heads, dim), dtype=dtype, device="cuda"), torch.empty_like(q.contiguous()), torch.empty_like(k.contiguous())
    r.apply(q, pos, q2, k=k, k_out=k2)
    two.append(k2, v, slots)
    before = copy_of(c)
    c.rotary_append(r, q, k, v, pos, slots, qo)
    assert torch.equal(qo, q2)
    assert torch.equal(bits(c.v), bits(two.v))
    if cache != F8:
        assert torch.equal(bits(c.k), bits(two.k))
        return
    assert torch.equal(c.v_scale, two.v_scale)
    take = [i for i in range(n) if 0 <= slots[i] < pages * page]
    at = slots[take]
    rest = torch.ones((pages * page,), dtype=torch.bool, device="cuda")
    rest[at] = False
    assert torch.equal(bits(by_slot(c, c.k)[rest]), bits(by_slot(before, before.k)[rest]))
    assert torch.equal(by_slot(c, c.k_scale)[rest], by_slot(before, before.k_scale)[rest])
    x, ang = values(k)[take], angles_of(r, pos)[take]
    want, e = decode.rotary(x, ang, layout == "half"), bound(x, ang, r)
    grid, sc = decode.scaled(want.reshape(-1, dim), 0, 448.0)
    off = (e.max(-1) / np.maximum(np.abs(want).max(-1), 2.0 ** -100)).reshape(-1, 1)
    assert np.all(np.abs(values(by_slot(c, c.k_scale)[at]).reshape(-1, 1) - sc) <= (4 * U + off) * sc)
    got = values(by_slot(c, c.k)[at].contiguous()).reshape(-1, dim)
    moved = (8 * U + off) * np.abs(grid) + e.reshape(-1, dim) / sc
    assert np.all(np.abs(got - grid) <= 0.5 * decode.e4m3_step(np.abs(grid) + moved) + moved)


def test_append_of_what_is_not_finite():
    g = gen(9)
    c = filled(g, 2, 4, 2, 64, F8, "head")
    r = A.Rotary.scaled(64)
    q, k, v = (normal(g, 2, 2, 64, dtype=torch.bfloat16) for _ in range(3))
    k[0, 1, 5], v[1, 0, 7] = float("inf"), float("nan")
    qo = torch.empty_like(q)
    c.rotary_append(r, q, k, v, torch.tensor([3, 4], device="cuda"), torch.tensor([0, 5], device="cuda"), qo)
    assert c.k_scale[0, 1, 0].isnan() and not c.k_scale[0, 0, 0].isnan() and c.v_scale[1, 0, 1].isnan()
    assert not bits(c.k[0, 1, 0]).any() and not bits(c.v[1, 0, 1]).any() and bits(c.k[0, 0, 0]).any()


def test_refusals_of_the_binding():
    g = gen(1)
    r = A.Rotary.scaled(64)
    q = normal(g, 2, 3, 64, dtype=torch.bfloat16)
    pos, o = torch.zeros((2,), dtype=torch.int64, device="cuda"), torch.empty_like(q)
    c = filled(g, 2, 4, 3, 64, torch.bfloat16, "head")
    for call in (lambda: r.apply(q, pos, o.float()), lambda: r.apply(q.cpu(), pos, o), lambda: r.apply(q, pos.int(), o),
                 lambda: r.apply(q, pos[:1], o), lambda: r.apply(q, pos, o, k=q), lambda: r.apply(q, pos, o, k_out=q),
                 lambda: r.apply(q.transpose(0, 1), pos, o), lambda: r.apply(q.float(), pos, o.float()),
                 lambda: r.apply(q[..., :60], pos, o[..., :60]), lambda: r.apply(q[0], pos, o[0]),
                 lambda: r.apply(q, pos, o, k=q[:, :, :56], k_out=o[:, :, :56]), lambda: r.apply(q[:0], pos[:0], o[:0]),
                 lambda: r.apply(q[..., :32], pos, o[..., :32]),
                 lambda: A.Rotary(r.frequencies.float()), lambda: A.Rotary(r.frequencies.cpu()), lambda: A.Rotary(r.frequencies[:0]),
                 lambda: A.Rotary(r.frequencies[::2]), lambda: A.Rotary(r.frequencies, layout="other"),
                 lambda: c.rotary_append(r, q, q[:, :2], q, pos, pos, o), lambda: c.rotary_append(r, q, q, q, pos, pos.int(), o),
                 lambda: c.rotary_append(r, q, q.half(), q, pos, pos, o), lambda: c.rotary_append(r, q.half(), q.half(), q.half(), pos, pos, o.half()),
                 lambda: c.rotary_append(r, q, q, q, pos, pos[:1], o)):
        with pytest.raises(A.AqmbError):
            call()
