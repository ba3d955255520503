"""Low-rank adapters where the kernels' loops are long (GPU): many steps of the inputs for few rows and for many, several outputs
a workgroup, odd and even numbers of the rank's steps. Random x, A and B everywhere, so that a step left out, taken twice or paired
with another's x shows. Tolerances are those of test_gpu_adapters.py, here for all rows of an adapter at once and
by sums in 64 bits on the GPU."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2606_12876_amd as A  # noqa: E402
from ops_helpers import U, gen, normal  # noqa: E402
from test_gpu_adapters import BF16, F16, F32, index_of, make  # noqa: E402

# binary digits behind the point and the least normal number's exponent
DIGITS = {BF16: (7, -126), F16: (10, -14), F32: (23, -126)}


def half_step(v, dtype):
    """Half the distance of a type's numbers at magnitude v (fp64, on the GPU)."""
    digits, least = DIGITS[dtype]
    return torch.exp2(torch.floor(torch.log2(v.clamp_min(2.0 ** least))).clamp_min(least) - digits - 1)


def check(ad, x, index, base, out):
    d = torch.float64
    want, e = base.to(d), torch.zeros(base.shape, dtype=d, device="cuda")
    none = (index < 0) | (index >= ad.n_adapters)
    for n in range(ad.n_adapters):
        rows = torch.nonzero(index == n)[:, 0]
        if not len(rows):
            continue
        r = ad.rank if ad.ranks is None else min(max(int(ad.ranks[n]), 0), ad.rank)
        if r == 0:
            continue
        a, b, xv, s = ad.a[n, :r].to(d), ad.b[n, :, :r].to(d), x[rows].to(d), ad.scales[n].to(d)
        t = s * (xv @ a.t())
        et = s * 2 * U * (ad.d_in / 32 + 64) * (xv.abs() @ a.abs().t()) + U * t.abs()
        et = et + (2.0 ** -24 * t.abs() if ad.dtype == BF16 else 2.0 ** -22 * (t.abs() + et).amax(1, keepdim=True))
        want[rows] += t @ b.t()
        e[rows] = et @ b.abs().t() + 2 * U * (3 * r / 32 + 33) * ((t.abs() + et) @ b.abs().t())
    e = e + 2 * U * (want.abs() + e)
    assert torch.equal(out[none], base[none])
    off = (out.to(d) - want).abs() - (e + half_step(want.abs() + e, out.dtype))
    off[none] = -1.0
    assert bool((off <= 0).all()), (off.max().item(), torch.nonzero(off > 0)[:5].tolist())


def run(ad, rows, index, out, odd=False, seed=0):
    """A call aside and in place, x from an odd element of its memory where asked for."""
    g = gen(seed)
    x = normal(g, rows * ad.d_in + odd, dtype=ad.dtype)[int(odd):].view(rows, ad.d_in)
    base = normal(g, rows, ad.d_out, dtype=out)
    y = torch.full_like(base, 7.0)
    ad.add(x, index, base, y)
    check(ad, x, index, base, y)
    z = base.clone()
    ad.add(x, index, z, z)
    assert torch.equal(z, y)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d_in,odd", [(11008, False), (11008, True), (9925, False), (14011, False), (20000, False)])
@pytest.mark.parametrize("rank", [16, 32, 64, 128, 200])
@pytest.mark.parametrize("rows,n", [(1, 1), (5, 3), (40, 26), (200, 2)])
def test_few_rows_of_many_inputs(rows, n, rank, d_in, odd, dtype):
    """Up to seven batches of loads a wave and a rest, by one workgroup a unit (1 and 5 rows) and by several (40 rows of 26 adapters)."""
    g = gen(rows + rank + d_in)
    ad = make(g, n, rank, d_in, 72, dtype)
    run(ad, rows, index_of(g, rows, n, False).clamp_min(0 if rows == 1 else -1), F32 if rows == 5 else dtype, odd, rank)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rank,ranks", [(64, [64, 40, 1]), (128, [33, 128, 65]), (256, [256, 130, 0])])
@pytest.mark.parametrize("rows", [3, 90, 400])
def test_mixed_ranks_of_many_inputs(rows, rank, ranks, dtype):
    """NaN behind the ranks."""
    g = gen(rows + rank)
    ad = make(g, 3, rank, 11008, 72, dtype, ranks)
    run(ad, rows, (torch.arange(rows, device="cuda") % 3).to(torch.int32), dtype, seed=rank)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rank", [16, 33, 64, 128, 200])
@pytest.mark.parametrize("rows,n,d_in", [(300, 5, 4099), (700, 3, 2305), (450, 40, 1100), (257, 1, 11008), (520, 2, 9925), (300, 4, 4095), (300, 4, 4032)])
def test_many_rows_of_many_inputs(rows, n, d_in, rank, dtype):
    """The inputs cut into parts, the last one with what is left of a step."""
    g = gen(rows + rank + d_in)
    ad = make(g, n, rank, d_in, 72, dtype)
    run(ad, rows, index_of(g, rows, n, rank % 2 == 0), dtype, d_in % 2 == 1 and rank == 64, rank)


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F16, F16), (BF16, F32), (F16, F32)])
@pytest.mark.parametrize("rank", [8, 16, 32, 40, 64, 96, 128, 161, 256])
@pytest.mark.parametrize("rows,d_out", [(2100, 4096), (2131, 4104), (2100, 4099), (2500, 3976)])
def test_several_outputs_a_workgroup(rows, d_out, rank, dtype, out):
    """256 outputs of a tile, a last workgroup's fewer: weights of the next outputs in the rank's last step, whose double buffer
    changes over within an output's steps or not."""
    g = gen(rows + rank)
    ad = make(g, 3, rank, 192, d_out, dtype)
    run(ad, rows, index_of(g, rows, 3, rank % 3 == 0), out, seed=rank)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_several_outputs_a_workgroup_with_mixed_ranks(dtype):
    g = gen(3)
    ad = make(g, 7, 128, 264, 4096, dtype, [128, 1, 0, 33, 64, 96, 127])
    run(ad, 3000, index_of(g, 3000, 7, False), dtype, seed=4)
    run(ad, 3000, index_of(g, 3000, 7, True), dtype, seed=5)


@pytest.mark.parametrize("rows", [2, 200, 300])
def test_a_large_stack_with_values_along_it(rows):
    """An adapter whose weights begin past 2^31 bytes: values at the start, around borders between parts of the inputs (an
    eighth of a quarter, few rows; a quarter, many), within them and at the end, zeros elsewhere. All sums are of 576 products."""
    g = gen(rows)
    n, rank, d = 3, 256, 3 * 2 ** 20
    part = d // 32
    at = torch.cat([torch.arange(i, i + 96, device="cuda") for i in (0, part - 50, 7 * part - 48, 16 * part - 33, 20 * part + 1001, d - 96)])
    a = torch.zeros((n, rank, d), dtype=BF16, device="cuda")
    assert a[2].storage_offset() * 2 > 2 ** 31
    a[2, :, at] = normal(g, rank, len(at), dtype=BF16, std=len(at) ** -0.5)
    x = torch.zeros((rows, d), dtype=BF16, device="cuda")
    x[:, at] = normal(g, rows, len(at), dtype=BF16)
    b, base = normal(g, n, 40, rank, dtype=BF16, std=rank ** -0.5), normal(g, rows, 40)
    got = torch.empty_like(base)
    A.Adapters(a, b).add(x, torch.full((rows,), 2, dtype=torch.int32, device="cuda"), base, got)
    small = A.Adapters(a[:, :, at].contiguous(), b, torch.ones((n,), device="cuda"))
    check(small, x[:, at].contiguous(), torch.full((rows,), 2, dtype=torch.int32, device="cuda"), base, got)
