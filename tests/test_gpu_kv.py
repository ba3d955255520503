"""Writing tokens into a paged cache and copying its pages (GPU). 16-bit caches are bit for bit; 8-bit ones
follow the scaling of aqmb_rms_norm: scales within 4 u, values within half a step of the e4m3 grid (and 8 u)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import decode

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2606_12876_amd as A  # noqa: E402
from ops_helpers import U, gen, normal, values  # noqa: E402

F8 = torch.float8_e4m3fn


def bits(t):
    return t.contiguous().view(torch.uint8)


def make(g, pages, page, kv, dim, dtype, layout):
    c = A.KVCache.allocate(pages, page, kv, dim, dtype, layout=layout)
    for t in (c.k, c.v):
        bits(t).copy_(torch.randint(0, 120, bits(t).shape, generator=g, device="cuda").to(torch.uint8))
    for t in (c.k_scale, c.v_scale):
        if t is not None:
            t.uniform_(0.5, 1.5, generator=g)
    return c


def by_slot(c, t):
    """[slots][kv](dim) view of a cache tensor in slot order."""
    t = t.transpose(1, 2) if c.layout == "head" else t
    return t.reshape(c.n_pages * c.page_size, c.n_kv_heads, *t.shape[3:])


@pytest.mark.parametrize("cache,dtype", [(torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16), (F8, torch.float16),
                                         (F8, torch.bfloat16)])
@pytest.mark.parametrize("layout", ["head", "slot"])
@pytest.mark.parametrize("n,pages,page,kv,dim", [(1, 3, 16, 2, 64), (5, 4, 1, 1, 8), (37, 9, 7, 3, 80), (64, 5, 20, 8, 128),
                                                 (20, 3, 8, 5, 256), (3, 2, 64, 1, 200)])
def test_append(n, pages, page, kv, dim, layout, cache, dtype):
    g = gen(n + dim)
    c = make(g, pages, page, kv, dim, cache, layout)
    n = min(n, pages * page)
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:n]
    qkv = normal(g, n, 3 * kv, dim, dtype=dtype)            # a fused projection's rows, one value wide of aligned
    k = torch.empty((n * 2 * kv * dim + 1,), dtype=dtype, device="cuda")[1:].view(n, 2 * kv, dim)[:, :kv]
    k.copy_(qkv[:, :kv])
    v = qkv[:, kv:2 * kv]
    v[0, 0] = 0.0
    slots_in = slots.clone()
    if n > 2:
        slots_in[1], slots_in[2] = -1, pages * page        # padding: skipped
    before = {name: by_slot(c, t).clone() for name, t in (("k", c.k), ("v", c.v))}
    scales = {name: None if t is None else by_slot(c, t).clone() for name, t in (("k", c.k_scale), ("v", c.v_scale))}
    c.append(k, v, slots_in)
    take = [i for i in range(n) if 0 <= slots_in[i] < pages * page]
    at = slots[take]
    rest = torch.ones((pages * page,), dtype=torch.bool, device="cuda")
    rest[at] = False
    for name, new, t, s in (("k", k, c.k, c.k_scale), ("v", v, c.v, c.v_scale)):
        now = by_slot(c, t)
        assert torch.equal(bits(now[rest]), bits(before[name][rest]))
        if cache != F8:
            assert torch.equal(bits(now[at]), bits(new[take].contiguous()))
            continue
        sn = by_slot(c, s)
        assert torch.equal(sn[rest], scales[name][rest])
        x = values(new[take])
        grid, want = decode.scaled(x.reshape(-1, dim), 0, 448.0)
        assert np.all(np.abs(values(sn[at]).reshape(-1, 1) - want) <= 4 * U * want)
        got = values(now[at].contiguous()).reshape(-1, dim)
        assert np.all(np.abs(got - grid) <= 0.5 * decode.e4m3_step(grid) + 8 * U * np.abs(grid))


def test_append_of_values_that_are_not_finite():
    g = gen(1)
    c = make(g, 2, 8, 2, 64, F8, "head")
    k, v = normal(g, 3, 2, 64, dtype=torch.bfloat16), normal(g, 3, 2, 64, dtype=torch.bfloat16)
    k[1, 0, 3], v[2, 1, 60] = float("nan"), float("-inf")
    c.append(k, v, torch.tensor([0, 5, 9], device="cuda"))
    ks, vs = by_slot(c, c.k_scale)[[0, 5, 9]], by_slot(c, c.v_scale)[[0, 5, 9]]
    assert torch.isnan(ks[1, 0]) and torch.isnan(vs[2, 1])
    assert torch.isfinite(ks).sum() == 5 and torch.isfinite(vs).sum() == 5
    assert (values(by_slot(c, c.k)[5, 0]) == 0).all() and (values(by_slot(c, c.v)[9, 1]) == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, F8])
@pytest.mark.parametrize("caches,pages,page,kv,dim,pairs", [(1, 3, 1, 1, 8, 1), (2, 9, 5, 3, 24, 4), (5, 30, 16, 8, 128, 15),
                                                            (64, 6, 8, 2, 64, 3), (1, 12, 64, 8, 128, 5)])
def test_copy_pages(caches, pages, page, kv, dim, pairs, dtype):
    g = gen(pages + dim)
    cs = [make(g, pages, page, kv, dim, dtype, "head" if dim % 16 else "slot") for _ in range(caches)]
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    dst, src = order[:pairs], order[pairs:][torch.randint(0, pages - pairs, (pairs,), generator=g, device="cuda")]
    src_in, dst_in = torch.cat((src, src[:3])), torch.cat((dst, torch.tensor([-1, pages, -9], device="cuda", dtype=torch.int32)[:len(src[:3])]))
    want = []
    for c in cs:
        for t in (c.k, c.v, c.k_scale, c.v_scale):
            if t is not None:
                w = t.clone()
                bits(w)[dst.long()] = bits(t)[src.long()]
                want.append((t, w))
    A.kv_copy_pages(cs, src_in, dst_in)
    for t, w in want:
        assert torch.equal(bits(t), bits(w))


def test_more_pairs_than_one_launch_takes():
    g = gen(7)
    n = 40000
    c = make(g, 2 * n, 1, 1, 8, torch.float16, "head")
    src = torch.arange(n, dtype=torch.int32, device="cuda")
    want = c.k[:n].clone()
    A.kv_copy_pages([c], src, src + n)
    assert torch.equal(bits(c.k[n:]), bits(want)) and torch.equal(bits(c.k[:n]), bits(want))


def test_copy_skips_a_page_onto_itself_and_bad_sources():
    g = gen(2)
    c = make(g, 5, 8, 2, 64, torch.float16, "head")
    want = c.k.clone()
    A.kv_copy_pages([c], torch.tensor([2, 7, -1], dtype=torch.int32, device="cuda"), torch.tensor([2, 0, 1], dtype=torch.int32, device="cuda"))
    assert torch.equal(bits(c.k), bits(want))


def test_pages_apart_and_beyond_32_bits():
    """Keys and values interleaved by page, pages past 2^32 elements."""
    kv, page, dim = 8, 128, 128
    n = (1 << 32) // (2 * kv * page * dim) + 4
    both = torch.empty((n, 2, kv, page, dim), dtype=torch.float16, device="cuda")
    c = A.KVCache(both[:, 0], both[:, 1])
    g = gen(3)
    both[n - 2:] = 0
    both[1:4] = normal(g, 3, 2, kv, page, dim, dtype=torch.float16)
    A.kv_copy_pages([c], torch.tensor([1, 3], dtype=torch.int32, device="cuda"), torch.tensor([n - 1, 0], dtype=torch.int32, device="cuda"))
    assert torch.equal(both[n - 1], both[1]) and torch.equal(both[0], both[3]) and (both[n - 2] == 0).all()
    k, v = normal(g, 2, kv, dim, dtype=torch.float16), normal(g, 2, kv, dim, dtype=torch.float16)
    c.append(k, v, torch.tensor([(n - 2) * page + 5, 5 * page], device="cuda"))
    assert torch.equal(both[n - 2, 0, :, 5], k[0]) and torch.equal(both[n - 2, 1, :, 5], v[0])
    both[n - 2, :, :, 5] = 0
    assert (both[n - 2] == 0).all() and torch.equal(both[5, 0, :, 0], k[1])


def test_pool_drives_a_cache():
    """Fork, copy on write, free and compaction with the pool's answers on a real cache: every sequence's keys stay
    what was appended to it."""
    g = gen(4)
    c, pool = A.KVCache.allocate(24, 8, 2, 64, torch.bfloat16), A.PagePool(24, 8, 8)
    text = {}

    def extend(s, n):
        slots, copies = pool.extend(s, n)
        if copies:
            A.kv_copy_pages([c], torch.tensor([copies[0][0]], dtype=torch.int32, device="cuda"),
                            torch.tensor([copies[0][1]], dtype=torch.int32, device="cuda"))
        k = normal(g, n, 2, 64, dtype=torch.bfloat16)
        c.append(k, -k, slots.cuda())
        text[s] = k if s not in text else torch.cat((text[s], k))

    def check():
        for s, want in text.items():
            t = pool.table(s).cuda().long()
            for x, w in ((c.k, want), (c.v, -want)):
                assert torch.equal(x[t].transpose(1, 2).reshape(-1, 2, 64)[:len(w)], w)

    a = pool.add()
    extend(a, 21)
    b = pool.fork(a)
    text[b] = text[a].clone()
    extend(b, 1)
    extend(a, 9)
    d = pool.fork(b)
    text[d] = text[b].clone()
    extend(d, 17)
    check()
    pool.free(a)
    del text[a]
    e = pool.add()
    extend(e, 8)
    pool.free(b)
    del text[b]
    pairs = pool.compact()
    if pairs:
        A.kv_copy_pages([c], torch.tensor([p[0] for p in pairs], dtype=torch.int32, device="cuda"),
                        torch.tensor([p[1] for p in pairs], dtype=torch.int32, device="cuda"))
    check()
    extend(d, 5)
    check()


def test_binding_refuses():
    g = gen(5)
    c = make(g, 4, 8, 2, 64, torch.bfloat16, "head")
    want = bits(c.k).clone()
    k, s = normal(g, 3, 2, 64, dtype=torch.bfloat16), torch.tensor([1, 2, 3], device="cuda")
    for a in ((k[:2], k, s), (k, k.half(), s), (k.half(), k.half(), s), (k, k, s.int()), (k, k[..., :32], s), (k, k, s.cpu()),
              (k.cpu(), k, s), (k[:0], k[:0], s[:0]), (k.transpose(1, 2).contiguous().transpose(1, 2), k, s)):
        with pytest.raises(A.AqmbError):
            c.append(*a)
    i = torch.tensor([0], dtype=torch.int32, device="cuda")
    other = make(g, 5, 8, 2, 64, torch.bfloat16, "head")
    for a in (([], i, i), ([c, other], i, i), ([c], i.long(), i), ([c], i, i[:0]), ([c], i[:0], i[:0]), ([c] * 65, i, i), ([c], i.cpu(), i)):
        with pytest.raises(A.AqmbError):
            A.kv_copy_pages(*a)
    torch.cuda.synchronize()
    assert torch.equal(bits(c.k), want)
