"""The decode step of examples/decode_step.py, all operators together, against the oracle in 64 bits (GPU).

The oracle keeps its own cache of what each stream has seen, exactly. Tolerance: about ten roundings to
bf16 (2^-9 each), an int8 rounding of the norm's output (half a step of 1/127 of the group's largest value,
about 0.4 % of the rows' size, whose ties fall differently after the roundings before it) and the rounding of
keys and values to the cache add up to less than 2 % of the output's norm; 3 % is allowed (4 % with the
8-bit cache, whose values are off by up to 1/16 of themselves, 2 % on average, in a sum over positions).
"""
from __future__ import annotations

import os
import sys

import numpy as np
import pytest
import torch

import oracle
from oracle import decode, formats

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2606_12876_amd as A  # noqa: E402
from ops_helpers import values  # noqa: E402

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from decode_step import Streams, random_block  # noqa: E402


def np_rotate(x, pos):
    half = x.shape[-1] // 2
    ang = pos * 10000.0 ** (-np.arange(half) / half)
    a, b = x[..., :half], x[..., half:]
    return np.concatenate((a * np.cos(ang) - b * np.sin(ang), b * np.cos(ang) + a * np.sin(ang)), -1)


class Reference:
    def __init__(self, block, raw):
        self.b, self.raw, self.seen = block, raw, {}

    def aq(self, name, x, k):
        codes, books, scales = self.raw[name]
        C = formats.f16_bits_to_f64(books.cpu().view(torch.int16).numpy().view(np.uint16))
        return oracle.linear(x, codes.cpu().numpy(), C, values(scales), k)

    def w4(self, name, x, d_in):
        w, s = self.raw[name]
        return x @ decode.w4_weights(w.cpu().numpy(), values(s), None, d_in, 32).T

    def step(self, h, k, streams):
        b = self.b
        x = decode.rms_norm(h, None, values(b.norms[0]), 0.0, b.eps)[1]
        q, kk, v = (self.aq(n, x, k).reshape(len(h), -1, b.dim) for n in "qkv")
        out = np.empty((len(h), b.heads, b.dim))
        for i, s in enumerate(streams):
            past = self.seen.setdefault(s, [])
            pos = len(past)
            past.append((np_rotate(kk[i], pos), v[i]))
            K, V = (np.stack([p[j] for p in past]) for j in (0, 1))
            for hd in range(b.heads):
                g = hd // (b.heads // b.kv_heads)
                out[i, hd] = decode.attend(np_rotate(q[i, hd], pos), K[:, g], V[:, g], b.dim ** -0.5)[0]
        a = self.aq("o", out.reshape(len(h), -1), k)
        h2, n2 = decode.rms_norm(a, h, values(b.norms[1]), 0.0, b.eps)
        grid, sc = decode.scaled(n2, 32, 127.0)
        x8 = np.rint(grid) * np.repeat(sc, 32, 1)[:, :n2.shape[1]]
        gate, up = self.w4("gate", x8, n2.shape[1]), self.w4("up", x8, n2.shape[1])
        m = gate / (1 + np.exp(-gate)) * up
        return h2 + self.w4("down", m, m.shape[1])


@pytest.mark.parametrize("cache,tol", [(torch.bfloat16, 0.03), (torch.float8_e4m3fn, 0.04)])
def test_decode_step_against_the_oracle(cache, tol):
    block, raw = random_block(cache_dtype=cache, seed=3)
    pool = A.PagePool(64, 16, 8)
    streams, ref = Streams(pool, [block.cache]), Reference(block, raw)
    rng = np.random.default_rng(0)
    live = [pool.add(), pool.add()]
    for step in range(40):
        if step == 21:                       # in the middle of a page
            live.append(pool.fork(live[0]))
            ref.seen[live[-1]] = list(ref.seen[live[0]])
        if step == 35:
            dead = live.pop(1)
            pool.free(dead)
            del ref.seen[dead]
            streams.copy(pool.compact())
        h = torch.from_numpy(rng.normal(size=(len(live), block.hidden))).bfloat16().cuda()
        k = 1 + step % 4
        got = block.step(h, k, *streams.advance(live))
        want = ref.step(values(h), k, live)
        err = np.linalg.norm(values(got) - want, axis=1) / np.linalg.norm(want, axis=1)
        assert np.all(err <= tol), (step, err)
