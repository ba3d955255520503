"""Scaling to 8 bits: the norm and the cache append do it alike, each step the rounded binary32 operation (GPU)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2606_12876_amd as A  # noqa: E402
from ops_helpers import gen, values  # noqa: E402

F8 = torch.float8_e4m3fn


def rows(n, cols, dtype):
    """Rows of multiples of 1/64 and for each the eps that makes mean(x^2) + eps 1, without a rounding on the way:
    the norm of such a row is the row."""
    g = gen(31)
    x = torch.randint(-60, 61, (n, cols), generator=g, device="cuda")
    x[:, 3] = torch.randint(61, 128, (n,), generator=g, device="cuda")          # the largest
    eps = 1.0 - (x.double() / 64).square().mean(1)
    assert (eps > 0).all()
    return (x.float() / 64).to(dtype), eps.tolist()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("cols", [64, 256])
def test_norm_and_append_scale_alike(cols, dtype):
    n = 150
    x, eps = rows(n, cols, dtype)
    w = torch.ones((cols,), dtype=dtype, device="cuda")
    xv = values(x).astype(np.float32)
    a = np.abs(xv).max(1, keepdims=True)
    want = {}
    for out, top in ((F8, np.float32(448)), (torch.int8, np.float32(127))):
        grid = xv * (top / a)
        assert grid.dtype == np.float32
        want[out] = (torch.from_numpy(grid).to(F8).view(torch.uint8) if out == F8 else
                     torch.from_numpy(np.rint(xv.astype(np.float64) * (top / a))).to(torch.int8), a / top)
        y, s = torch.empty((n, cols), dtype=out, device="cuda"), torch.empty((n, 1), device="cuda")
        for i in range(n):
            A.rms_norm(x[i:i + 1], w, y[i:i + 1], eps=eps[i], scales=s[i:i + 1])
        assert np.array_equal(s.cpu().numpy(), want[out][1])
        assert torch.equal(y.view(torch.uint8 if out == F8 else out).cpu(), want[out][0])
    c = A.KVCache.allocate(n, 1, 1, cols, F8)
    c.append(x.view(n, 1, cols), -x.view(n, 1, cols), torch.arange(n, device="cuda"))
    assert torch.equal(c.k.view(torch.uint8).view(n, cols).cpu(), want[F8][0])
    assert np.array_equal(values(c.v), -values(c.k))
    for s in (c.k_scale, c.v_scale):
        assert np.array_equal(s.view(n, 1).cpu().numpy(), want[F8][1])
