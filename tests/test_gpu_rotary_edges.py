"""Rotary positions: the bits of what is not turned (GPU)."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2606_12876_amd as A  # noqa: E402
from ops_helpers import gen, normal  # noqa: E402
from test_gpu_rotary import LAYOUTS  # noqa: E402


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dim,rot", [(8, 2), (16, 12), (24, 16), (80, 22), (64, 32), (200, 100)])
@pytest.mark.parametrize("tokens", [1, 40])
def test_values_behind_the_pairs_keep_their_bits(tokens, dim, rot, layout, dtype):
    """Every bit pattern, NaNs with their payloads and subnormal values among them, alone and in a cache of the same type; 40
    tokens of small heads are more than one workgroup's."""
    each = dim - rot
    heads = -(-65536 // (each * tokens))
    q = normal(gen(dim), tokens, heads, dim, dtype=dtype)
    bits = torch.arange(tokens * heads * each, device="cuda").view(tokens, heads, each) % 65536
    q.view(torch.int16)[..., rot:] = bits.to(torch.int16)
    r = A.Rotary.scaled(rot, layout=layout)
    pos = torch.arange(tokens, device="cuda") + 3
    out = torch.zeros_like(q)
    r.apply(q, pos, out)
    assert torch.equal(out.view(torch.int16)[..., rot:], q.view(torch.int16)[..., rot:])
    assert out[..., :rot].isfinite().all() and not torch.equal(out[..., :rot], q[..., :rot])
    c = A.KVCache.allocate(tokens, 1, heads, dim, dtype)
    c.rotary_append(r, q, q, q, pos, torch.arange(tokens, device="cuda"), torch.empty_like(q))
    assert torch.equal(c.k.view(torch.int16).view(q.shape), out.view(torch.int16))
    assert torch.equal(c.v.view(torch.int16).view(q.shape), q.view(torch.int16))
