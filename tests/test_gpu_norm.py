"""aqmb_rms_norm against the oracle in 64 bits (GPU).

Tolerance: h is one binary32 addition; the sum of squares adds at most 32 values in a thread and then
at most 22 partial sums (6 exchanges, 16 waves), so its relative error is below 60 u (u = 2^-24), half
of that after the root; the division, root and three products add less than 10 u. Together
|v' - v| <= 64 u |v| (h counted with the additions' |x| + |r|), and the output one rounding more. On
the 8-bit grid the scale's two roundings join: 70 u of the value, and half a step of the grid.
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

H16 = [torch.float16, torch.bfloat16]


def check(x, r, w, w0, eps, y, r2, scales, group):
    xv, rv = values(x), None if r is None else values(r)
    h, v = decode.rms_norm(xv, rv, values(w), w0, eps)
    # the part of v's error that cancellation in x + r leaves: u (|x| + |r|) of h, carried to v
    amp = np.abs(v) if r is None else np.abs(v) + np.abs(v) / np.maximum(np.abs(h), 1e-300) * (np.abs(xv) + np.abs(rv)) / 64
    if r is not None:
        assert np.all(np.abs(values(r2) - h) <= half_ulp(h, x.dtype) + 2 * U * np.abs(h))
    if scales is None:
        assert np.all(np.abs(values(y) - v) <= half_ulp(v, y.dtype) + 64 * U * amp)
        return
    top = decode.LARGEST["f8" if y.dtype == torch.float8_e4m3fn else "i8"]
    grid, s = decode.scaled(v, group, top)
    assert np.all(np.abs(values(scales) - s) <= 70 * U * s)
    step = decode.e4m3_step(grid) if y.dtype == torch.float8_e4m3fn else 1.0
    gamp = np.abs(grid) / np.maximum(np.abs(v), 1e-300) * amp + np.abs(grid)
    assert np.all(np.abs(values(y) - grid) <= 0.5 * step + 70 * U * gamp)
    assert np.max(np.abs(values(y))) <= top


@pytest.mark.parametrize("dtype", H16)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 8), (1, 9), (9, 64), (4, 127), (2, 128), (7, 511), (3, 513),
                                       (2, 1024), (5, 1025), (1, 2048), (3, 2049), (2, 4096), (3, 4097), (1, 8191),
                                       (2, 8200), (1, 11008), (2, 16384), (1, 16385), (2, 32768)])
def test_norm_and_residual(rows, cols, dtype):
    g = gen(rows * 40000 + cols)
    x, r, w = normal(g, rows, cols, dtype=dtype), normal(g, rows, cols, dtype=dtype), normal(g, cols, dtype=dtype, std=0.3)
    for res in (None, r):
        for out in (dtype, torch.float32):
            y = torch.full((rows, cols), 7.0, dtype=out, device="cuda")
            r2 = None if res is None else torch.full_like(x, 7.0)
            A.rms_norm(x, w, y, eps=1e-5, weight_offset=1.0, residual=res, residual_out=r2)
            check(x, res, w, 1.0, 1e-5, y, r2, None, 0)


@pytest.mark.parametrize("dtype", H16)
@pytest.mark.parametrize("out", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (5, 33), (2, 129), (6, 500), (2, 1000), (3, 2305), (1, 4096),
                                       (2, 9000), (1, 20001)])
def test_eight_bits(rows, cols, group, out, dtype):
    g = gen(rows * 40000 + cols + group)
    x, r, w = normal(g, rows, cols, dtype=dtype), normal(g, rows, cols, dtype=dtype), normal(g, cols, dtype=dtype)
    x[0, cols // 2] *= 50.0
    y = torch.empty((rows, cols), dtype=out, device="cuda")
    s = torch.empty((rows, -(-cols // group) if group else 1), device="cuda")
    r2 = torch.empty_like(x)
    A.rms_norm(x, w, y, eps=1e-6, residual=r, residual_out=r2, scales=s, scale_group=group)
    check(x, r, w, 0.0, 1e-6, y, r2, s, group)


def test_zero_rows_and_small_groups():
    x = torch.zeros((3, 96), dtype=torch.bfloat16, device="cuda")
    x[1, 40] = 1.0
    w = torch.ones((96,), dtype=torch.bfloat16, device="cuda")
    for out, top in ((torch.float8_e4m3fn, 448.0), (torch.int8, 127.0)):
        y, s = torch.full((3, 96), 1, device="cuda").to(out), torch.empty((3, 3), device="cuda")
        A.rms_norm(x, w, y, eps=1e-6, scales=s, scale_group=32)
        got, want = values(y), np.zeros((3, 96))
        want[1, 40] = top
        assert np.array_equal(got, want)
        sv = values(s)
        assert np.all(sv[[0, 0, 0, 1, 1, 2], [0, 1, 2, 0, 2, 1]] == np.float32(2.0 ** -100) / np.float32(top))
        assert sv[1, 1] > 0.01
    y = torch.empty((3, 96), dtype=torch.bfloat16, device="cuda")
    A.rms_norm(x[:1], w, y[:1], eps=0.0)            # 0 * (1 / 0): the formula's NaN
    assert torch.isnan(y[0]).all()


def test_values_that_are_not_finite():
    x = torch.ones((4, 256), dtype=torch.float16, device="cuda")
    x[1, 70], x[2, 5] = float("nan"), float("inf")
    w = torch.ones((256,), dtype=torch.float16, device="cuda")
    y = torch.empty_like(x)
    A.rms_norm(x, w, y, eps=1e-6)
    yv = values(y)
    assert np.all(yv[[0, 3]] == 1) and np.all(np.isnan(yv[1]))
    assert np.isnan(yv[2, 5]) and np.all(np.delete(yv[2], 5) == 0)      # inf * 0, and 1 / inf elsewhere
    w[200] = float("inf")                                              # one column, one group of every row
    for out in (torch.float8_e4m3fn, torch.int8):
        q, s = torch.ones((4, 256), device="cuda").to(out), torch.empty((4, 4), device="cuda")
        A.rms_norm(x, w, q, eps=1e-6, scales=s, scale_group=64)
        sv, qv = values(s), values(q)
        assert np.all(np.isnan(sv[:, 3])) and np.all(qv[:, 192:] == 0)
        assert np.all(np.isfinite(sv[0, :3])) and np.all(qv[0, :192] == (448 if out != torch.int8 else 127))
        assert np.all(np.isnan(sv[1])) and np.all(qv[1] == 0)
        assert np.isnan(sv[2, 0]) and np.all(np.isfinite(sv[2, 1:3])) and np.all(qv[2] == 0)


@pytest.mark.parametrize("out", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("size", [3e38, 1e38, 1e-20, 1e-29])
def test_large_and_small_groups(size, out):
    """Groups whose largest magnitude has a subnormal reciprocal, or is close to the scales' floor."""
    g = gen(8)
    x = torch.where(torch.rand((2, 256), generator=g, device="cuda") < 0.5, -1.0, 1.0).bfloat16()
    w = (size * torch.rand((256,), generator=g, device="cuda")).bfloat16()
    y, s = torch.empty((2, 256), dtype=out, device="cuda"), torch.empty((2, 4), device="cuda")
    A.rms_norm(x, w, y, eps=0.0, scales=s, scale_group=64)
    check(x, None, w, 0.0, 0.0, y, None, s, 64)


@pytest.mark.parametrize("dtype", H16)
def test_strides_alignment_and_in_place(dtype):
    g = gen(5)
    for cols, off in ((300, 1), (1027, 3), (4096, 5)):
        big = normal(g, 5, cols + 37, dtype=dtype)
        x, r = big[:, off:off + cols], normal(g, 5, cols + 11, dtype=dtype)[:, 2:2 + cols]
        w = normal(g, cols + 1, dtype=dtype)[1:]
        want, want_r = torch.empty((5, cols), dtype=dtype, device="cuda"), torch.empty((5, cols), dtype=dtype, device="cuda")
        A.rms_norm(x.contiguous(), w.clone(), want, eps=1e-6, residual=r.contiguous(), residual_out=want_r)
        wide = torch.full((5, cols + 9), 3.0, dtype=dtype, device="cuda")
        r2 = torch.full((5, cols + 11), 4.0, dtype=dtype, device="cuda")
        A.rms_norm(x, w, wide[:, 4:4 + cols], eps=1e-6, residual=r, residual_out=r2[:, 2:2 + cols])
        assert torch.equal(wide[:, 4:4 + cols], want) and torch.equal(r2[:, 2:2 + cols], want_r)
        assert (wide[:, :4] == 3).all() and (wide[:, 4 + cols:] == 3).all()           # nothing beside the rows
        assert (r2[:, :2] == 4).all() and (r2[:, 2 + cols:] == 4).all()
        q8, s = torch.full((5, cols + 3), 9, dtype=torch.int8, device="cuda"), torch.empty((5, -(-cols // 32)), device="cuda")
        A.rms_norm(x, w, q8[:, 1:1 + cols], eps=1e-6, scales=s, scale_group=32)
        q2, s2 = torch.empty((5, cols), dtype=torch.int8, device="cuda"), torch.empty_like(s)
        A.rms_norm(x.contiguous(), w, q2, eps=1e-6, scales=s2, scale_group=32)
        assert torch.equal(q8[:, 1:1 + cols], q2) and torch.equal(s, s2) and (q8[:, 0] == 9).all() and (q8[:, cols + 1:] == 9).all()
        xc, rc = x.contiguous(), r.contiguous()                                         # in place
        A.rms_norm(xc, w, xc, eps=1e-6, residual=rc, residual_out=rc)
        assert torch.equal(xc, want) and torch.equal(rc, want_r)
        xc, y = x.contiguous(), torch.empty_like(want)                                  # the sum over x
        A.rms_norm(xc, w, y, eps=1e-6, residual=r.contiguous(), residual_out=xc)
        assert torch.equal(y, want) and torch.equal(xc, want_r)


def test_offsets_beyond_32_bits():
    """Rows 2^26 elements apart: the last one starts past 2^31 elements (4 GiB)."""
    n, pitch, cols = 34, 1 << 26, 1000
    flat = torch.empty(((n - 1) * pitch + cols,), dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((n, cols), (pitch, 1))
    src = normal(gen(6), n, cols, dtype=torch.bfloat16)
    x.copy_(src)
    w = torch.ones((cols,), dtype=torch.bfloat16, device="cuda")
    y, want = torch.empty_like(src), torch.empty_like(src)
    A.rms_norm(x, w, y, eps=1e-6)
    A.rms_norm(src, w, want, eps=1e-6)
    assert torch.equal(y, want)
    A.rms_norm(src, w, x, eps=1e-6)
    assert torch.equal(x, want)


def test_binding_refuses():
    x = torch.zeros((2, 64), dtype=torch.bfloat16, device="cuda")
    w, y = x[0].clone(), torch.full_like(x, 5.0)
    bad = [dict(weight=w[:63]), dict(weight=w.half()), dict(y=y[:1]), dict(y=y[:, :63]), dict(x=x[0]), dict(x=x.float()),
           dict(residual=x), dict(residual_out=x), dict(residual=x, residual_out=x.half()),
           dict(residual=x[:, :32], residual_out=x[:, :32]), dict(scales=torch.zeros((2, 2), device="cuda"), scale_group=32),
           dict(y=x.t().contiguous().t()), dict(x=x.cpu()), dict(y=torch.zeros((2, 64), dtype=torch.int8, device="cuda")),
           dict(y=torch.zeros((2, 64), dtype=torch.int8, device="cuda"), scales=torch.zeros((2, 1), device="cuda"), scale_group=32),
           dict(y=torch.zeros((2, 64), dtype=torch.int32, device="cuda"))]
    for kw in bad:
        a = dict(x=x, weight=w, y=y)
        a.update(kw)
        with pytest.raises(A.AqmbError):
            A.rms_norm(a.pop("x"), a.pop("weight"), a.pop("y"), eps=1e-6, **a)
    torch.cuda.synchronize()
    assert (y == 5).all()
