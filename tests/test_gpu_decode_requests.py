"""A decode step with adapters beside q and v, rotary positions on the way into the cache and log probabilities at the
end, all operators together, against the oracle in 64 bits (GPU).

Tolerances as in the test of the step without them: about ten roundings to bf16 and one to int8, 3 % of the output's norm (4 % with the
8-bit cache); the adapters' own addition rounds once more, to bf16. The log probabilities are checked against the oracle on the
logits that were answered, to the binary32 of their sums: 2^-24 (vocab / 64 + 128) of what is summed, about 2e-5 for 1000 tokens."""
from __future__ import annotations

import os
import sys

import numpy as np
import pytest
import torch

from oracle import decode

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2606_12876_amd as A  # noqa: E402
from ops_helpers import gen, normal, values  # noqa: E402
from test_gpu_decode_step import Reference  # noqa: E402

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from decode_step import Streams, answer, random_adapters, random_block  # noqa: E402


class WithAdapters(Reference):
    index = None

    def aq(self, name, x, k):
        y = super().aq(name, x, k)
        ad = self.b.adapters.get(name)
        if ad is not None:
            y = y + decode.adapted(x, self.index, values(ad.a), values(ad.b), values(ad.scales), [ad.rank] * ad.n_adapters)
        return y


@pytest.mark.parametrize("cache,tol", [(torch.bfloat16, 0.03), (torch.float8_e4m3fn, 0.04)])
def test_a_step_with_all_that_requests_bring(cache, tol):
    block, raw = random_block(cache_dtype=cache, seed=5)
    plain = block.adapters
    block.adapters = random_adapters(block, seed=2)
    pool = A.PagePool(64, 16, 8)
    streams, ref = Streams(pool, [block.cache]), WithAdapters(block, raw)
    live = [pool.add() for _ in range(5)]
    g = gen(4)
    head = normal(g, block.hidden, 1000, dtype=torch.bfloat16, std=0.1)
    for step in range(12):
        h = normal(g, len(live), block.hidden, dtype=torch.bfloat16)
        ref.index = [s % 5 - 1 for s in live]
        index = torch.tensor(ref.index, dtype=torch.int32, device="cuda")
        out = block.step(h, 4, *streams.advance(live), index=index)
        want = ref.step(values(h), 4, live)
        err = np.linalg.norm(values(out) - want, axis=1) / np.linalg.norm(want, axis=1)
        assert err.max() < tol, (step, err)
        t = torch.randint(0, 1000, (len(live),), generator=g, device="cuda")
        lp, entropy, ids, tops = answer(out, head, t)
        z = values(out @ head)
        for i in range(len(live)):
            p, _, e = decode.log_probs(z[i])
            assert abs(float(lp[i]) - p[t[i]]) <= 2e-5 * (1 + abs(p[t[i]])) and abs(float(entropy[i]) - e) <= 2e-5 * (1 + e)
            best = np.argsort(-z[i], kind="stable")[:3]
            assert np.array_equal(ids[i].cpu().numpy(), best) and np.allclose(tops[i].cpu().numpy(), p[best], rtol=2e-5, atol=2e-5)
        if step == 6:
            streams.free(live.pop(2))
    assert plain == {}
    # without an index the adapters stay out
    a, b = Streams(pool, [block.cache]), normal(g, len(live), block.hidden, dtype=torch.bfloat16)
    args = a.advance(live)
    one = block.step(b, 4, *args)
    none = torch.full((len(live),), -1, dtype=torch.int32, device="cuda")
    assert torch.equal(one, block.step(b, 4, *args, index=none))
