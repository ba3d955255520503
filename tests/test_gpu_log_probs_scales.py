"""Log probabilities at the largest scales (GPU). Tolerances as in test_gpu_log_probs.py."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2606_12876_amd as A  # noqa: E402
from test_gpu_log_probs import check, run  # noqa: E402


@pytest.mark.parametrize("scale", [2.0 ** 100, 2.0 ** 127, 2.3e38])
def test_the_largest_scales(scale):
    """The factor of the exponents, scale / log 2, is finite up to 2.35e38."""
    z = torch.tensor([[1e-38, 0.0, -1e-38, 2e-38], [-1.0, -2.0, 3.0, 2.5], [0.0, 0.0, -0.0, 0.0]], device="cuda")
    z[1] *= 2.0 ** -126
    t = torch.tensor([[0, 3], [2, 1], [1, 0]], device="cuda")
    check(z, t, run(z, t, 4, scale=scale), scale=scale)


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_scales_whose_factor_overflows_are_refused(scale):
    """They made every row of finite logits one of NaN."""
    z, lse = torch.zeros((2, 30), device="cuda"), torch.full((2,), 7.0, device="cuda")
    with pytest.raises(A.AqmbError, match="scale"):
        A.log_probs(z, lse=lse, scale=scale)
    assert (lse == 7.0).all()
