"""Rotary positions of many tokens, alone and into a cache (GPU): to the bit what the same tokens give in small calls, which
test_gpu_rotary.py holds against the oracle; some tokens against the oracle themselves.

Many: 131072 heads of up to 64 values, 65536 of up to 128, 32768 of more, and at most 256, 128 and 64 heads a token. Those calls are cut
into several tokens a workgroup where a token has few heads, loaded four heads at a time, and stored past the caches."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2606_12876_amd as A  # noqa: E402
from ops_helpers import gen, normal, values  # noqa: E402
from test_gpu_rotary import F8, LAYOUTS, angles_of, bits, check, copy_of, filled  # noqa: E402


def many(n, total, dim):
    """Whether a call is one of many heads, as above."""
    at_once = 64 if dim <= 64 else 32 if dim <= 128 else 16
    return n * total >= 2048 * at_once and total <= 4 * at_once


def in_small(n, total, call):
    """call(slice of tokens) for all of them, few at a time, an odd number."""
    step = max(1, 30000 // total) | 1
    for i in range(0, n, step):
        call(slice(i, min(i + step, n)))


# heads of queries and of keys; 0: none
SHAPES = [(3001, 40, 4, 64, 64), (131077, 1, 0, 64, 32), (65543, 1, 1, 24, 16), (2801, 48, 0, 64, 48), (700, 190, 66, 40, 10), (6007, 8, 3, 96, 48), (3003, 21, 3, 128, 20), (520, 100, 28, 128, 128),
          (8200, 5, 3, 80, 32), (65537, 1, 0, 128, 128), (5003, 5, 2, 200, 22), (1025, 60, 4, 256, 256), (2049, 9, 9, 256, 100), (32771, 1, 0, 136, 136)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("n,heads,kv,dim,rot", SHAPES)
def test_many_tokens(n, heads, kv, dim, rot, layout, dtype):
    assert many(n, heads + kv, dim)
    g = gen(n)
    r = A.Rotary.scaled(rot, layout=layout, scaling=A.RotaryScaling.RAMP, factor=4.0, original_length=512)
    rows = normal(g, n, heads + kv + 1, dim, dtype=dtype)                # one head beside them that stays
    q, k = rows[:, :heads], rows[:, heads:heads + kv]
    pos = torch.randint(-1000, 100000, (n,), generator=g, device="cuda")
    for inverse in (False, True):
        want, got = ((torch.empty((n, heads, dim), dtype=dtype, device="cuda"), torch.zeros((n, kv, dim), dtype=dtype, device="cuda")) for _ in range(2))
        call = lambda s, qo, ko: r.apply(q[s], pos[s], qo[s], k=k[s] if kv else None, k_out=ko[s] if kv else None, inverse=inverse)  # noqa: E731
        in_small(n, heads + kv, lambda s: call(s, *want))
        call(slice(0, n), *got)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    some = torch.randperm(n, generator=g, device="cuda")[:12]
    some = torch.cat((some, torch.tensor([0, 1, n - 1], device="cuda")))
    check(got[0][some], values(q[some]), angles_of(r, pos[some]), r, dtype, inverse)
    kept = rows[:, -1].clone()
    r.apply(q, pos, q, k=k if kv else None, k_out=k if kv else None, inverse=True)          # in place
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(rows[:, -1], kept)


@pytest.mark.parametrize("n,heads,kv,dim", [(700, 200, 100, 64), (400, 150, 20, 128), (500, 60, 10, 256)])
def test_tokens_of_more_heads_than_a_workgroup_takes(n, heads, kv, dim):
    """As many heads in all, but too many of a token: the way of few tokens."""
    assert n * (heads + kv) >= 32768 and not many(n, heads + kv, dim)
    g = gen(n)
    r = A.Rotary.scaled(dim)
    q, k, pos = normal(g, n, heads, dim, dtype=torch.bfloat16), normal(g, n, kv, dim, dtype=torch.bfloat16), torch.arange(n, device="cuda")
    out, ko = torch.empty_like(q), torch.empty_like(k)
    r.apply(q, pos, out, k=k, k_out=ko)
    some = torch.tensor([0, n // 2, n - 1], device="cuda")
    check(out[some], values(q[some]), angles_of(r, pos[some]), r, torch.bfloat16)
    check(ko[some], values(k[some]), angles_of(r, pos[some]), r, torch.bfloat16)


@pytest.mark.parametrize("cache,dtype", [(torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16), (F8, torch.float16), (F8, torch.bfloat16)])
@pytest.mark.parametrize("order", ["head", "slot"])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("n,page,heads,kv,dim,rot", [
    (3001, 16, 40, 4, 64, 64), (45001, 20, 1, 1, 64, 32), (1400, 7, 32, 32, 40, 10), (6007, 16, 5, 3, 96, 48), (2501, 64, 21, 3, 128, 20), (2100, 1, 16, 8, 128, 128),
    (8200, 16, 2, 3, 80, 32), (5003, 33, 3, 2, 200, 22), (1025, 16, 24, 4, 256, 256), (1300, 8, 9, 9, 256, 100)])
def test_a_prompt_into_the_cache(n, page, heads, kv, dim, rot, layout, order, cache, dtype):
    """Some slots skipped; what no token is written to stays."""
    total = heads + 2 * kv
    assert many(n, total, dim)
    g = gen(n + dim)
    pages = -(-n // page) + 3
    c = filled(g, pages, page, kv, dim, cache, order)
    r = A.Rotary.scaled(rot, layout=layout)
    rows = normal(g, n, total, dim, dtype=dtype)
    q, k, v = rows[:, :heads], rows[:, heads:heads + kv], rows[:, heads + kv:]
    pos = 100 + torch.arange(n, device="cuda")
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:n].clone()
    slots[::17], slots[5], slots[n - 2] = -1, pages * page, 2 ** 40
    small, want, got = copy_of(c), torch.empty((n, heads, dim), dtype=dtype, device="cuda"), torch.empty((n, heads, dim), dtype=dtype, device="cuda")
    in_small(n, total, lambda s: small.rotary_append(r, q[s], k[s], v[s], pos[s], slots[s], want[s]))
    c.rotary_append(r, q, k, v, pos, slots, got)
    assert torch.equal(got, want)
    for a, b in ((c.k, small.k), (c.v, small.v), (c.k_scale, small.k_scale), (c.v_scale, small.v_scale)):
        assert a is None or torch.equal(bits(a), bits(b))
    some = torch.randperm(n, generator=g, device="cuda")[:8]
    check(got[some], values(q[some]), angles_of(r, pos[some]), r, dtype)
    c.rotary_append(r, q, k, v, pos, slots, q)                               # the queries in place
    assert torch.equal(q, want)
    for a, b in ((c.k, small.k), (c.v, small.v), (c.k_scale, small.k_scale), (c.v_scale, small.v_scale)):
        assert a is None or torch.equal(bits(a), bits(b))
