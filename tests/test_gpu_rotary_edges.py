"""Rotary positions at angles far beyond a turn, and the bits of what is not turned (GPU)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2606_12876_amd as A  # noqa: E402
from ops_helpers import U, gen, half_ulp, normal, values  # noqa: E402
from oracle import decode  # noqa: E402
from test_gpu_rotary import LAYOUTS, angles_of, partner  # noqa: E402


@pytest.mark.parametrize("layout", LAYOUTS)
def test_angles_of_any_size(layout):
    """The angle is the binary64 product of the position and the frequency, as the oracle's, and sine and cosine are within 2^-22 of
    its own whatever its size: the tolerance of test_gpu_rotary.py without a term that grows with the angle."""
    g = gen(15)
    r = A.Rotary(torch.tensor([1.0, 0.75, 1 / 3, 10000.0 ** -0.25, 1e-3, 6.283185307179586, 1e-9, 4000.5], dtype=torch.float64, device="cuda"), layout=layout)
    edge = [2 ** p + d for p in (20, 27, 30, 31, 32, 40, 48, 52, 53, 60, 62) for d in (-1, 0, 1)] + [10 ** 6, 10 ** 9, 10 ** 12, 2 ** 63 - 1, -2 ** 63]
    pos = torch.tensor(edge + [-p for p in edge[:-1]], device="cuda")
    q = normal(g, len(pos), 3, 16, dtype=torch.float16)
    out = torch.empty_like(q)
    for inverse in (False, True):
        r.apply(q, pos, out, inverse=inverse)
        x, ang = values(q), angles_of(r, pos)
        want = decode.rotary(x, -ang if inverse else ang, layout == "half")
        e = partner(x, 8, layout == "half") * (2.0 ** -22 + 4 * U)
        off = np.abs(values(out) - want) - (e + half_ulp(np.abs(want) + e, torch.float16))
        assert np.all(off <= 0), [(edge[i % len(edge)], o) for i, o in enumerate(off.max((1, 2))) if o > 0]


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
