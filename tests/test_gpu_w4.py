"""The product with 4-bit group-scaled weights against the oracle in 64 bits (GPU).

Tolerance. In a group of g inputs the products are exact and summed in binary32 (int8: exactly), with
a magnitude of at most T_g = s sum (q + z + 32) |x| (32: the offset that bf16 operands carry, twice), so
each group is off by at most 2 g u T_g (u = 2^-24); the groups' sums, at most their number plus 16 waves of
them, add (groups + 16) u sum_g |group|; the scale's products 4 u. The output adds one rounding.
Integer inputs whose every partial sum fits in 24 bits have to come out exactly.
"""
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

F8, I8 = torch.float8_e4m3fn, torch.int8
XT = [torch.float16, torch.bfloat16, F8, I8]


def layer(g, d_out, d_in, group, zeros, ints=False):
    n = -(-d_in // group)
    w = torch.randint(0, 256, (d_out, (d_in + 1) // 2), generator=g, device="cuda").to(torch.uint8)
    if ints:
        s = 2.0 ** torch.randint(-1, 2, (d_out, n), generator=g, device="cuda").float()
    else:
        s = 0.004 * (0.5 + torch.rand((d_out, n), generator=g, device="cuda"))
    z = torch.randint(0, 16, (d_out, n), generator=g, device="cuda").to(torch.uint8) if zeros else None
    return w, s.half(), z


def inputs(g, batch, d_in, xt, group, ints=False):
    """x of type xt and, for 8 bits, its scales by group."""
    if ints:
        x = torch.randint(-4, 5, (batch, d_in), generator=g, device="cuda").float()
    else:
        x = normal(g, batch, d_in) * (30.0 if xt in (F8, I8) else 1.0)
    if xt == I8:
        x = x.round().clamp(-127, 127)
    if xt == F8:
        x = x.clamp(-448, 448)
    xs = None
    if xt in (F8, I8):
        xs = torch.rand((batch, -(-d_in // group)), generator=g, device="cuda") + 0.5
        if ints:
            xs = 2.0 ** torch.randint(-1, 2, xs.shape, generator=g, device="cuda").float()
    return x.to(xt), xs


def reference(x, xs, w, s, z, d_in, group):
    """(y, bound without the output's rounding), both fp64."""
    xv, sv = values(x), values(s)
    per = np.arange(d_in) // group
    if xs is not None:
        sx = values(xs)
        xv = xv * (sx[:, per] if sx.shape[1] > 1 else sx)
    W = decode.w4_weights(w.cpu().numpy(), sv, None if z is None else z.cpu().numpy(), d_in, group)
    q = decode.nibbles(w.cpu().numpy(), d_in)
    zv = 8.0 if z is None else values(z)[:, per]
    n = sv.shape[1]
    y, bound = xv @ W.T, np.zeros((xv.shape[0], W.shape[0]))
    T = np.abs(xv) @ ((q + zv + 32.0) * sv[:, per]).T
    parts = np.zeros_like(bound)
    for j in range(n):
        a = slice(j * group, (j + 1) * group)
        parts += np.abs(xv[:, a] @ W[:, a].T)
    bound = 2 * group * U * T + (n + 20) * U * parts + 4 * U * np.abs(y)
    return y, bound


def run(x, xs, w, s, z, d_in, group, out):
    lin = A.W4Linear(w, s, z, d_in=d_in, group_size=group)
    y = torch.full((x.shape[0], w.shape[0]), float("nan"), dtype=out, device="cuda")
    lin.gemv(x, y, xs)
    got = values(y)
    lin.close()
    return got


SIZES = [(1, 1), (16, 128), (17, 127), (5, 33), (64, 32), (33, 130), (100, 257), (31, 640), (257, 1000), (40, 2313),
         (1000, 72), (130, 4096)]


@pytest.mark.parametrize("xt", XT)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("d_out,d_in", SIZES)
def test_random(d_out, d_in, group, xt):
    g = gen(d_out * 5000 + d_in + group)
    for batch, zeros, out in ((1, False, torch.float32), (2, True, torch.float16), (7, True, torch.float32),
                              (16, False, torch.bfloat16)):
        w, s, z = layer(g, d_out, d_in, group, zeros)
        x, xs = inputs(g, batch, d_in, xt, group)
        y, bound = reference(x, xs, w, s, z, d_in, group)
        got = run(x, xs, w, s, z, d_in, group, out)
        assert np.all(np.abs(got - y) <= bound + half_ulp(y, out)), (batch, np.max(np.abs(got - y) / bound))


@pytest.mark.parametrize("xt", XT)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("d_out,d_in", [(4097, 2200), (4200, 300), (8209, 2100), (8209, 200), (12305, 1111), (16401, 2313)])
def test_tall_layers(d_out, d_in, group, xt):
    """Workgroups of one to four row tiles and of 8 to 16 waves, the last of them partly outside: every output
    is written, some rows are held against the formula."""
    g = gen(d_out + d_in + group)
    rows = torch.tensor(sorted(set(range(40)) | set(range(0, d_out, 101)) | set(range(d_out - 70, d_out))), device="cuda")
    for batch, zeros, out in ((1, True, torch.float32), (3, False, torch.bfloat16), (16, True, torch.float32)):
        w, s, z = layer(g, d_out, d_in, group, zeros)
        x, xs = inputs(g, batch, d_in, xt, group)
        y, bound = reference(x, xs, w[rows], s[rows], z[rows] if zeros else None, d_in, group)
        got = run(x, xs, w, s, z, d_in, group, out)
        assert np.isfinite(got).all()
        got = got[:, rows.cpu().numpy()]
        assert np.all(np.abs(got - y) <= bound + half_ulp(y, out)), (batch, np.max(np.abs(got - y) / bound))


@pytest.mark.parametrize("xt", XT)
@pytest.mark.parametrize("d_out,d_in,group", [(1, 1, 32), (19, 77, 32), (48, 512, 64), (100, 1111, 128), (33, 2048, 128),
                                              (520, 3001, 64)])
def test_integers_come_out_exactly(d_out, d_in, group, xt):
    g = gen(d_in + 9)
    for batch, zeros in ((1, True), (5, False), (16, True)):
        w, s, z = layer(g, d_out, d_in, group, zeros, ints=True)
        x, xs = inputs(g, batch, d_in, xt, group, ints=True)
        y, _ = reference(x, xs, w, s, z, d_in, group)
        assert np.max(np.abs(y)) < 2 ** 22
        assert np.array_equal(run(x, xs, w, s, z, d_in, group, torch.float32), y)


@pytest.mark.parametrize("xt", XT)
def test_sums_keep_binary32(xt):
    """The bounds above are worst cases; on random data the error is a walk. A group's partial sums are
    about 24 sqrt(g) against a result of about 4.6 sqrt(g) and see 4 to 8 roundings, so the result is off by about
    24 / 4.6 * sqrt(8) u = 15 u in the 2-norm; 64 u is allowed. (Sums of 17 bits would give 128 u and more.)"""
    g = gen(21)
    w, s, z = layer(g, 300, 2048, 128, True)
    x, xs = inputs(g, 8, 2048, xt, 128)
    y, _ = reference(x, xs, w, s, z, 2048, 128)
    err = run(x, xs, w, s, z, 2048, 128, torch.float32) - y
    assert np.linalg.norm(err) <= 64 * U * np.linalg.norm(y)


@pytest.mark.parametrize("xt", [F8, I8])
def test_one_scale_per_row(xt):
    g = gen(12)
    w, s, z = layer(g, 100, 500, 64, True)
    x, _ = inputs(g, 6, 500, xt, 64)
    xs = torch.rand((6, 1), generator=g, device="cuda") + 0.5
    y, bound = reference(x, xs, w, s, z, 500, 64)
    assert np.all(np.abs(run(x, xs, w, s, z, 500, 64, torch.float32) - y) <= bound + half_ulp(y, torch.float32))


@pytest.mark.parametrize("xt", XT)
def test_extreme_operands(xt):
    """Subnormal and largest x: the nibbles are read as subnormals, which must not be flushed."""
    g = gen(3)
    d_in = 256
    w, s, z = layer(g, 48, d_in, 128, True, ints=True)
    big, tiny = {torch.float16: (60000.0, 2.0 ** -24), torch.bfloat16: (2.0 ** 100, 2.0 ** -110), F8: (448.0, 2.0 ** -9),
                 I8: (-127.0, 1.0)}[xt]
    x = torch.where(torch.rand((4, d_in), generator=g, device="cuda") < 0.5, tiny, 0.0)
    x[2:] = x[2:] / tiny * big
    x = x.to(xt)
    xs = torch.ones((4, 2), device="cuda") if xt in (F8, I8) else None
    y, bound = reference(x, xs, w, s, z, d_in, 128)
    got = run(x, xs, w, s, z, d_in, 128, torch.float32)
    assert np.all(np.isfinite(got)) and np.any(got[0] != 0)
    assert np.all(np.abs(got - y) <= bound + half_ulp(y, torch.float32))


@pytest.mark.parametrize("xt", [torch.float16, torch.bfloat16])
def test_not_finite(xt):
    """A row of x that is not finite spoils its own outputs and no others."""
    g = gen(4)
    w, s, z = layer(g, 40, 300, 64, False)
    x, _ = inputs(g, 5, 300, xt, 64)
    want = run(x, None, w, s, z, 300, 64, torch.float32)
    x[1, 299], x[3, 17] = float("nan"), float("inf")
    got = run(x, None, w, s, z, 300, 64, torch.float32)
    assert not np.isfinite(got[[1, 3]]).any() and np.array_equal(got[[0, 2, 4]], want[[0, 2, 4]])


def test_strides_and_alignment():
    g = gen(8)
    for xt in XT:
        w, s, z = layer(g, 50, 200, 32, True)
        x, xs = inputs(g, 7, 200, xt, 32)
        lin = A.W4Linear(w, s, z, d_in=200, group_size=32)
        want, wide = torch.empty((7, 50), device="cuda"), torch.full((7, 61), 3.0, device="cuda")
        lin.gemv(x, want, xs)
        store = torch.zeros((7, 213), dtype=torch.int8, device="cuda").to(xt) if xt in (F8, I8) else \
            torch.full((7, 213), float("nan"), dtype=xt, device="cuda")
        store[:, 3:203] = x
        lin.gemv(store[:, 3:203], wide[:, 5:55], xs)
        assert torch.equal(wide[:, 5:55], want) and (wide[:, :5] == 3).all() and (wide[:, 55:] == 3).all()
        lin.close()


def test_results_do_not_depend_on_the_other_rows():
    g = gen(9)
    w, s, z = layer(g, 700, 1500, 128, True)
    x, _ = inputs(g, 16, 1500, torch.bfloat16, 128)
    full = run(x, None, w, s, z, 1500, 128, torch.float32)
    for b in (1, 2, 5, 11):
        assert np.array_equal(run(x[:b], None, w, s, z, 1500, 128, torch.float32), full[:b])


def test_layer_class_and_refusals():
    g = gen(10)
    w, s, z = layer(g, 24, 96, 32, True)
    lin = A.W4Linear(w, s, z, group_size=32)
    assert (lin.d_in, lin.d_out) == (96, 24)
    d = A.w4_get_desc(lin.handle)
    assert (d.d_out, d.d_in, d.group_size) == (24, 96, 32)
    x = normal(g, 2, 3, 96, dtype=torch.float16)
    y = lin(x)
    assert y.shape == (2, 3, 24) and y.dtype == torch.float16
    y2 = torch.empty((6, 24), dtype=torch.float16, device="cuda")
    A.w4_gemv(lin.handle, x.reshape(6, 96), y2)
    assert torch.equal(y.reshape(6, 24), y2)
    y2.fill_(5)
    x = x.reshape(6, 96)
    q = torch.zeros((6, 96), dtype=I8, device="cuda")
    for a in ((x[:, :95], y2), (x, y2[:5]), (x, y2[:, :23]), (x.float(), y2), (x, y2.to(I8)), (q, y2), (x, y2, torch.ones((6, 1), device="cuda")),
              (q, y2, torch.ones((6, 2), device="cuda")), (x.cpu(), y2), (x.t().contiguous().t(), y2),
              (torch.zeros((17, 96), dtype=torch.float16, device="cuda"), torch.zeros((17, 24), device="cuda")),
              (torch.zeros((0, 96), dtype=torch.float16, device="cuda"), torch.zeros((0, 24), device="cuda"))):
        with pytest.raises(A.AqmbError):
            lin.gemv(*a)
    torch.cuda.synchronize()
    assert (y2 == 5).all()
    h = lin.handle
    lin.close()
    with pytest.raises(A.AqmbError):
        A.w4_gemv(h, x, y2)
    for bad in ((w[:, :47], s, z), (w, s[:, :2], z), (w, s, z[:, :2]), (w, s.float(), z), (w.to(torch.int8), s, z)):
        with pytest.raises(A.AqmbError):
            A.W4Linear(*bad, d_in=96, group_size=32)


@pytest.mark.parametrize("xt", [torch.bfloat16, F8, I8])
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("zero", [None, 0, 255])
def test_largest_inputs(zero, group, xt):
    """|X| = 2^112 throughout, of one sign in some rows, with the largest and smallest weights and zero points: every
    sum stays finite and as exact as ever."""
    g = gen(13)
    d_out, d_in = 40, 300
    w, s, z = layer(g, d_out, d_in, group, zero is not None)
    w[:16], w[16:32] = 0xFF, 0
    if zero is not None:
        z.fill_(zero)
    sign = torch.where(torch.rand((3, d_in), generator=g, device="cuda") < 0.5, -1.0, 1.0)
    sign[1], sign[2] = 1.0, -1.0
    xs = None
    if xt == torch.bfloat16:
        x = (sign * 2.0 ** 112).to(xt)
    else:
        top = {F8: 448.0, I8: 127.0}[xt]
        x, xs = (sign * top).to(xt), torch.full((3, -(-d_in // group)), 2.0 ** 112 / top * (1 - 2.0 ** -23), device="cuda")
    y, bound = reference(x, xs, w, s, z, d_in, group)
    got = run(x, xs, w, s, z, d_in, group, torch.float32)
    assert np.all(np.isfinite(got)) and np.all(np.abs(got - y) <= bound + half_ulp(y, torch.float32))
