"""Paged attention of one token against the oracle in 64 bits (GPU).

Tolerance. A score is off by at most d = 2 D u scale sum |q||k| + 8 u |score| (binary32 sums of exact
products; u = 2^-24), the running maximum's rescalings and the exponential by a few u more, so the
weights are off by a factor within 1 +- 2 (max d + 32 u); they enter the product in two 16-bit parts
(2^-16); sums over n positions add 2 n u. All of it multiplies A = sum_t w_t |V_t|:
  |out' - out| <= (4 (max d + 32 u) + 2^-15 + 4 n u) A + half a spacing of the output.
lse: |error| <= 2 max d + 64 u + 4 u |lse| + 2 n u.
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

F8 = torch.float8_e4m3fn


def build(g, lens, kv, dim, page, dtype, cache_dtype=None, layout="head", spare=3, fill=float("nan"), per=None):
    """A cache whose slots hold `fill` where no sequence has a token, page tables in random order with
    entries that no length reaches set to numbers that are no page."""
    n = len(lens)
    per = per or max(1, max(-(-t // page) for t in lens) + 1)
    used = [-(-t // page) for t in lens]
    total = sum(used) + spare
    order = torch.randperm(total, generator=g, device="cuda").tolist()
    table = torch.full((n, per), 2 ** 31 - 1, dtype=torch.int32)
    table[:, ::2] = -5
    shape = (total, kv, page) if layout == "head" else (total, page, kv)
    k, v = normal(g, *shape, dim), normal(g, *shape, dim)
    ks = vs = None
    held = torch.zeros((total, page), dtype=torch.bool)
    for i, t in enumerate(lens):
        for p in range(used[i]):
            table[i, p] = order.pop()
            held[table[i, p], :min(page, t - p * page)] = True
    free = (~held).cuda()
    free = free[:, None, :] if layout == "head" else free[:, :, None]
    if cache_dtype == F8:
        ks, vs = (0.01 * (0.5 + torch.rand(shape, generator=g, device="cuda")) for _ in range(2))
        k, v = ((x * 100).clamp(-448, 448).to(F8) for x in (k, v))
        ks.masked_fill_(free, fill)
        vs.masked_fill_(free, fill)
        if np.isnan(fill):
            k, v = (torch.where(free[..., None], torch.tensor(0x7F, dtype=torch.uint8, device="cuda"), x.view(torch.uint8)).view(F8)
                    for x in (k, v))
    else:
        k, v = (x.to(dtype).masked_fill_(free[..., None], fill) for x in (k, v))
    return A.KVCache(k, v, ks, vs, layout=layout), table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")


def stored(c):
    k, v = values(c.k), values(c.v)
    if c.k_scale is not None:
        k, v = k * values(c.k_scale)[..., None], v * values(c.v_scale)[..., None]
    return k, v


def check(c, q, table, lens, scale, window, out, lse):
    k, v = stored(c)
    if c.layout == "slot":
        k, v = k.transpose(0, 2, 1, 3), v.transpose(0, 2, 1, 3)
    qv, got, ls = values(q), values(out), None if lse is None else values(lse)
    tab, n, heads = table.cpu().numpy(), q.shape[0], q.shape[1]
    per = heads // c.n_kv_heads
    for i, t in enumerate(lens.tolist()):
        pos = np.arange(max(0, t - window) if window else 0, t)
        page, slot = tab[i, pos // c.page_size], pos % c.page_size
        ok = (page >= 0) & (page < c.n_pages)
        page, slot = page[ok], slot[ok]
        for h in range(heads):
            K, V = k[page, h // per, slot], v[page, h // per, slot]
            ref, rl = decode.attend(qv[i, h], K, V, scale)
            if len(K) == 0:
                assert np.all(got[i, h] == 0), (i, h)
                assert ls is None or ls[i, h] == -np.inf
                continue
            s = K @ qv[i, h] * scale
            w = np.exp(s - rl)
            d = np.max(2 * c.head_dim * U * abs(scale) * (np.abs(K) @ np.abs(qv[i, h])) + 8 * U * np.abs(s))
            bound = (4 * (d + 32 * U) + 2.0 ** -15 + 4 * len(K) * U) * (w @ np.abs(V)) + half_ulp(ref, q.dtype)
            err = np.abs(got[i, h] - ref)
            assert np.all(err <= bound), (i, h, t, np.max(err / bound))
            if ls is not None:
                assert abs(ls[i, h] - rl) <= 2 * d + 64 * U + 4 * U * abs(rl) + 2 * len(K) * U, (i, h)


def attend(c, q, table, lens, scale=None, window=0, max_length=None, with_lse=True):
    out = torch.full_like(q, 9.0)
    lse = torch.full(q.shape[:2], 9.0, device="cuda") if with_lse else None
    scale = q.shape[2] ** -0.5 if scale is None else scale
    c.attention(q, table, lens, out, scale=scale, window=window, max_length=max_length, lse=lse)
    check(c, q, table, lens, scale, window, out, lse)
    return out


LENS = [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257]


@pytest.mark.parametrize("dtype,cache", [(torch.float16, None), (torch.bfloat16, None), (torch.float16, F8), (torch.bfloat16, F8)])
@pytest.mark.parametrize("layout", ["head", "slot"])
@pytest.mark.parametrize("page", [1, 7, 8, 16, 20, 64, 100, 512])
def test_lengths_and_pages(page, layout, dtype, cache):
    g = gen(page)
    c, table, lens = build(g, LENS, 2, 64, page, dtype, cache, layout)
    q = normal(g, len(LENS), 6, 64, dtype=dtype, std=2.0)
    attend(c, q, table, lens)


@pytest.mark.parametrize("dtype,cache", [(torch.float16, None), (torch.bfloat16, None), (torch.bfloat16, F8)])
@pytest.mark.parametrize("dim", [8, 16, 24, 40, 64, 72, 80, 96, 120, 128, 136, 160, 192, 200, 248, 256])
def test_head_dims(dim, dtype, cache):
    g = gen(dim)
    c, table, lens = build(g, [150, 1, 40], 3, dim, 16, dtype, cache)
    attend(c, normal(g, 3, 6, dim, dtype=dtype, std=2.0), table, lens)


@pytest.mark.parametrize("kv,heads", [(1, 1), (1, 2), (3, 9), (2, 14), (1, 16), (2, 32), (1, 17), (1, 33), (2, 80), (1, 128), (8, 8)])
def test_head_layouts(kv, heads):
    g = gen(heads)
    c, table, lens = build(g, [300, 0, 77], kv, 128, 32, torch.bfloat16)
    attend(c, normal(g, 3, heads, 128, dtype=torch.bfloat16), table, lens)
    c, table, lens = build(g, [130], kv, 256, 32, torch.float16, F8, "slot")
    attend(c, normal(g, 1, heads, 256, dtype=torch.float16), table, lens)


@pytest.mark.parametrize("window", [1, 2, 8, 31, 32, 33, 100, 128, 129, 1000])
@pytest.mark.parametrize("page", [8, 20])
def test_window(window, page):
    """Pages that lie wholly before the window may have been given to others: their entries are no pages."""
    g = gen(window)
    lens_ = [0, 1, 31, 32, 33, 100, 129, 400, 777]
    c, table, lens = build(g, lens_, 2, 64, page, torch.bfloat16)
    q = normal(g, len(lens_), 4, 64, dtype=torch.bfloat16)
    attend(c, q, table, lens, window=window)
    for i, t in enumerate(lens_):
        table[i, :max(0, t - window) // page] = -1
    attend(c, q, table, lens, window=window)


@pytest.mark.parametrize("dtype,cache", [(torch.bfloat16, None), (torch.float16, F8)])
def test_long_and_ragged(dtype, cache):
    g = gen(77)
    lens_ = [20001, 0, 1, 4097, 12345]
    c, table, lens = build(g, lens_, 1, 128, 64, dtype, cache)
    q = normal(g, 5, 4, 128, dtype=dtype, std=2.0)
    out = attend(c, q, table, lens)
    # a sequence's result does not depend on the others, only on max_length
    one = torch.empty_like(q[:1])
    for i in (0, 3, 4):
        c.attention(q[i:i + 1], table[i:i + 1], lens[i:i + 1], one, scale=128 ** -0.5, max_length=20001)
        ref = values(out[i:i + 1])
        assert np.all(np.abs(values(one) - ref) <= 2 * half_ulp(ref, dtype) + 1e-4 * np.max(np.abs(ref)))


@pytest.mark.parametrize("dtype,cache", [(torch.float16, None), (torch.bfloat16, None), (torch.bfloat16, F8)])
@pytest.mark.parametrize("layout", ["head", "slot"])
@pytest.mark.parametrize("dim", [8, 64, 72, 128, 136, 256])
def test_split_sequences(dim, layout, dtype, cache):
    """Chunks that are full, partly full and empty, joined: many of them, and two or three of each sequence."""
    g = gen(dim + 1)
    lens_ = [1030, 0, 1, 128, 129, 700]
    c, table, lens = build(g, lens_, 2, dim, 20, dtype, cache, layout)
    q = normal(g, len(lens_), 6, dim, dtype=dtype, std=2.0)
    assert c.workspace_bytes(6, len(lens_), 1030) > 0
    attend(c, q, table, lens, max_length=1030)
    attend(c, q, table, lens, max_length=1030, window=1028)
    lens_ = [1100, 0, 1, 384, 512, 513, 1025] + [64] * 25
    c, table, lens = build(g, lens_, 8, dim, 20, dtype, cache, layout)
    attend(c, normal(g, len(lens_), 8, dim, dtype=dtype, std=2.0), table, lens)


@pytest.mark.parametrize("kv,per", [(1, 17), (3, 2), (5, 1), (6, 20), (12, 1), (16, 3)])
@pytest.mark.parametrize("dim", [8, 24, 64, 80])
@pytest.mark.parametrize("cache", [None, F8])
def test_heads_that_share_lines(cache, dim, kv, per):
    """Every (sequence, head, chunk) is done once where heads lie side by side and do not fill cache lines."""
    g = gen(100 * kv + dim)
    lens_ = [1030, 3, 0, 400, 77]
    c, table, lens = build(g, lens_, kv, dim, 16, torch.float16, cache, "slot")
    q = normal(g, 5, kv * per, dim, dtype=torch.float16, std=2.0)
    attend(c, q, table, lens)
    attend(c, q[1:], table[1:], lens[1:], max_length=400)


def test_many_short_sequences():
    g = gen(90)
    lens_ = [i % 4 for i in range(5000)]
    c, table, lens = build(g, lens_, 2, 16, 2, torch.bfloat16)
    q = normal(g, 5000, 4, 16, dtype=torch.bfloat16)
    out = torch.full_like(q, 9.0)
    c.attention(q, table, lens, out, scale=0.25)
    pick = list(range(0, 5000, 61)) + [4999]
    check(c, q[pick], table[pick], lens[pick], 0.25, 0, out[pick], None)
    assert (out[torch.tensor(lens_) == 0] == 0).all()


def test_split_counts_agree():
    """The same sequence under bounds that split it differently."""
    g = gen(78)
    c, table, lens = build(g, [999], 2, 64, 16, torch.float16, per=8000)
    q = normal(g, 1, 8, 64, dtype=torch.float16)
    for bound in (999, 1000, 5000, 128000):
        attend(c, q, table, lens, max_length=bound)


def test_lengths_are_clamped():
    g = gen(79)
    c, table, lens = build(g, [40, 40, 40], 1, 64, 16, torch.bfloat16)
    q = normal(g, 3, 2, 64, dtype=torch.bfloat16)
    odd = torch.tensor([1000000, -3, 40], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    c.attention(q, table, odd, out, scale=0.1, max_length=40)
    check(c, q, table, torch.tensor([40, 0, 40]), 0.1, 0, out, None)


def test_pages_that_do_not_exist_are_skipped():
    g = gen(80)
    c, table, lens = build(g, [100, 64, 300], 2, 128, 16, torch.float16)
    table[0, 2], table[1, :4], table[2, 0], table[2, 18] = c.n_pages, -1, -1, 2 ** 30
    attend(c, normal(g, 3, 4, 128, dtype=torch.float16), table, lens)


def test_sharp_and_flat_softmax():
    g = gen(81)
    for dtype in (torch.float16, torch.bfloat16):
        c, table, lens = build(g, [700, 129], 1, 64, 16, dtype)
        q = normal(g, 2, 4, 64, dtype=dtype)
        attend(c, q, table, lens, scale=0.0)
        attend(c, q, table, lens, scale=-0.3)
        attend(c, q * 30, table, lens, scale=1.0)
        # one position far above many that are small together: the small ones must not be lost
        c.k.zero_()
        c.v.fill_(1.0)
        c.k[table[0, 0], 0, 0] = 1.0
        q.fill_(1.0)
        attend(c, q, table, lens, scale=15.0 * 0.6931 / 64)
        attend(c, q, table, lens, scale=20.0 * 0.6931 / 64)


def test_scores_that_are_not_finite():
    g = gen(82)
    c, table, lens = build(g, [50, 50], 1, 64, 16, torch.bfloat16)
    q = normal(g, 2, 3, 64, dtype=torch.bfloat16)
    want = attend(c, q, table, lens)
    c.v[table[0, 1], 0, 3, 5] = float("inf")              # one value of sequence 0
    out = torch.empty_like(q)
    c.attention(q, table, lens, out, scale=64 ** -0.5)
    assert torch.isinf(out[0, :, 5]).all() and torch.equal(out[1], want[1])
    keep = [d for d in range(64) if d != 5]
    assert torch.equal(out[0][:, keep], want[0][:, keep])
    c.k[table[0, 2], 0, 0, 0] = float("nan")              # one key of sequence 0
    c.attention(q, table, lens, out, scale=64 ** -0.5)
    assert torch.isnan(out[0]).all() and torch.equal(out[1], want[1])


@pytest.mark.parametrize("cache_dtype", [None, F8])
@pytest.mark.parametrize("length", [40, 900, 40000])      # one workgroup, a few chunks, many
def test_a_score_that_is_nan_shows_in_the_denominator(length, cache_dtype):
    g = gen(85)
    c, table, lens = build(g, [length, length], 1, 128, 16, torch.float16, cache_dtype)
    q = normal(g, 2, 3, 128, dtype=torch.float16)
    out, lse = torch.empty_like(q), torch.empty((2, 3), device="cuda")
    c.attention(q, table, lens, out, scale=128 ** -0.5, lse=lse)
    assert torch.isfinite(lse).all()
    want, stats = out.clone(), lse.clone()
    q[0, 1, 7] = float("nan")                             # one head of sequence 0
    c.attention(q, table, lens, out, scale=128 ** -0.5, lse=lse)
    assert torch.isnan(out[0, 1]).all() and torch.isnan(lse[0, 1])
    q[0, 1, 7] = 0.0
    if cache_dtype is None:                               # and one key, for every head
        c.k[table[0, 2], 0, 0, 0] = float("nan")
    else:
        c.k_scale[table[0, 2], 0, 0] = float("nan")
    c.attention(q, table, lens, out, scale=128 ** -0.5, lse=lse)
    assert torch.isnan(out[0]).all() and torch.isnan(lse[0]).all()
    assert torch.equal(out[1], want[1]) and torch.equal(lse[1], stats[1])


def test_strides():
    g = gen(83)
    lens_ = [70, 33, 5]
    c, table, lens = build(g, lens_, 2, 64, 16, torch.bfloat16)
    q = normal(g, 3, 4, 64, dtype=torch.bfloat16)
    want = attend(c, q, table, lens)
    # q inside a wider row (a fused projection's output), out likewise, a wider table, pages apart
    qkv = torch.full((3, 8, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    qkv[:, 2:6] = q
    wide = torch.full((3, 6, 64), 4.0, dtype=torch.bfloat16, device="cuda")
    big = torch.full((3, table.shape[1] + 7), -9, dtype=torch.int32, device="cuda")
    big[:, :table.shape[1]] = table
    both = torch.full((c.n_pages, 2, 2, 16, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    both[:, 0], both[:, 1] = c.k, c.v
    c2 = A.KVCache(both[:, 0], both[:, 1])
    c2.attention(qkv[:, 2:6], big[:, :table.shape[1]], lens, wide[:, 1:5], scale=64 ** -0.5)
    # (the split follows the table's width, which is the same here)
    assert torch.equal(wide[:, 1:5], want) and (wide[:, 0] == 4).all() and (wide[:, 5] == 4).all()


def test_offsets_beyond_32_bits():
    """Pages past 2^32 elements of the cache (8 GiB each of keys and values)."""
    kv, page, dim = 8, 128, 128
    n = (1 << 32) // (kv * page * dim) + 40
    k = torch.empty((n, kv, page, dim), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    g = gen(84)
    order = [n - 1, 3, n - 20, n - 2]
    small = A.KVCache(normal(g, 4, kv, page, dim, dtype=torch.bfloat16), normal(g, 4, kv, page, dim, dtype=torch.bfloat16))
    for i, p in enumerate(order):
        k[p], v[p] = small.k[i], small.v[i]
    c = A.KVCache(k, v)
    q, lens = normal(g, 1, 16, dim, dtype=torch.bfloat16), torch.tensor([500], dtype=torch.int32, device="cuda")
    t1, t2 = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in ([0, 1, 2, 3], order))
    want, got = torch.empty_like(q), torch.empty_like(q)
    small.attention(q, t1, lens, want, scale=0.1)
    c.attention(q, t2, lens, got, scale=0.1)
    assert torch.equal(got, want)
    check(small, q, t1, lens, 0.1, 0, want, None)


def test_workspace_is_checked_and_used():
    g = gen(85)
    c, table, lens = build(g, [900], 1, 64, 16, torch.float16, per=200)      # the bound, not the length, splits
    q = normal(g, 1, 2, 64, dtype=torch.float16)
    want = attend(c, q, table, lens)
    need = c.workspace_bytes(2, 1, table.shape[1] * 16)
    assert need > 0
    out = torch.full_like(q, 5.0)
    ws = torch.full((need // 4 + 64,), float("nan"), device="cuda")
    with pytest.raises(A.AqmbError):
        c.attention(q, table, lens, out, scale=0.125, workspace=ws.view(torch.uint8)[:need - 4])
    torch.cuda.synchronize()
    assert (out == 5).all()
    c.attention(q, table, lens, out, scale=64 ** -0.5, workspace=ws[:need // 4])
    assert torch.equal(out, want) and torch.isnan(ws[need // 4:]).all()


@pytest.mark.parametrize("stream", [False, True])
def test_a_workspace_that_is_not_dense_is_refused(stream):
    """An expanded or strided tensor has fewer bytes of its own than its number of elements says."""
    g = gen(87)
    c, table, lens = build(g, [1300], 2, 64, 16, torch.float16)
    q = normal(g, 1, 2, 64, dtype=torch.float16)
    need = c.workspace_bytes(2, 1, table.shape[1] * 16)
    out = torch.full_like(q, 5.0)
    base = torch.full((need,), 7, dtype=torch.uint8, device="cuda")
    kw = dict(stream=torch.cuda.current_stream()) if stream else {}
    for ws in (base[:1].expand(need), torch.stack((base, base), 1)[:, 0]):
        with pytest.raises(A.AqmbError, match="dense"):
            c.attention(q, table, lens, out, scale=0.125, workspace=ws, **kw)
    torch.cuda.synchronize()
    assert (out == 5).all() and (base == 7).all()


def test_binding_refuses():
    g = gen(86)
    c, table, lens = build(g, [20, 20], 2, 64, 16, torch.bfloat16)
    q = normal(g, 2, 4, 64, dtype=torch.bfloat16)
    out = torch.full_like(q, 5.0)
    ok = dict(q=q, page_table=table, lengths=lens, out=out, scale=0.1)
    bad = [dict(q=q[0]), dict(q=q[..., :32]), dict(q=q.half(), out=out.half()), dict(q=q[:, :3], out=out[:, :3]), dict(out=out[:1]),
           dict(out=out.float()), dict(page_table=table[:1]), dict(page_table=table.long()), dict(page_table=table[0]),
           dict(lengths=lens.long()), dict(lengths=lens[:1]), dict(max_length=10 ** 6), dict(max_length=-1), dict(window=-1),
           dict(lse=torch.zeros((2, 3), device="cuda")), dict(lengths=lens.cpu()), dict(scale=float("nan")),
           dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(q=q[:0], out=out[:0], lengths=lens[:0], page_table=table[:0])]
    for kw in bad:
        a = {**ok, **kw}
        with pytest.raises(A.AqmbError):
            c.attention(a.pop("q"), a.pop("page_table"), a.pop("lengths"), a.pop("out"), **a)
    torch.cuda.synchronize()
    assert (out == 5).all()
    k = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    s = torch.zeros((4, 2, 16), device="cuda")
    for a, kw in (((k, k[:3]), {}), ((k, k.half()), {}), ((k.float(), k.float()), {}), ((k.transpose(1, 2), k.transpose(1, 2)), {}),
                  ((k, k, s, s), {}), ((k.to(F8), k.to(F8)), {}), ((k.to(F8), k.to(F8), s, s[:3]), {}), ((k, k), dict(layout="x")),
                  ((k[:1].expand(4, 2, 16, 64), k[:1].expand(4, 2, 16, 64)), {}), ((k.cpu(), k.cpu()), {})):
        with pytest.raises(A.AqmbError):
            A.KVCache(*a, **kw)


@pytest.mark.parametrize("below", [8, 18, 24, 26, 27, 28, 34, 40, 60, 200])
@pytest.mark.parametrize("length,page,per", [(300, 16, None), (1300, 16, None), (40000, 16, None), (9000, 4096, 512)])
@pytest.mark.parametrize("dtype,cache", [(torch.float16, None), (torch.bfloat16, None), (torch.float16, F8)])
def test_small_weights_before_large_values(dtype, cache, length, page, per, below):
    """One position far above the others (by `below` units of the natural logarithm), whose value is a ten-millionth
    of theirs: what each of the others weighs must neither be lost nor grow. A sequence whole, in few chunks, in many,
    and in the largest chunks, where a wave takes 32 tiles one after the other."""
    g = gen(91)
    c, table, lens = build(g, [length], 1, 64, page, dtype, cache, per=per)
    held = [(int(table[0, t // page]), t % page) for t in (0, length // 2, length - 1)]
    q = torch.ones((1, 3, 64), dtype=dtype, device="cuda")
    for p, slot in held:
        c.k.view(torch.uint8).zero_()
        c.v.copy_(torch.where(torch.rand(c.v.shape, generator=g, device="cuda") < 0.7, 256.0, -128.0).to(c.v.dtype))
        c.k[p, 0, slot] = 1.0
        if cache is None:
            c.v.mul_(48.0)
            c.v[p, 0, slot] = 0.001
        else:
            c.k_scale.fill_(1.0), c.v_scale.fill_(48.0)
            c.v[p, 0, slot] = 1.0
            c.v_scale[p, 0, slot] = 0.001
        attend(c, q, table, lens, scale=below / 64.0)


@pytest.mark.parametrize("length", [40, 300, 1300, 40000])
def test_weights_of_zero_and_infinite_values(length):
    """fp16: a value of infinity gives infinity, scores of -infinity give weights of zero, and nothing else counts."""
    g = gen(92)
    c, table, lens = build(g, [length], 1, 64, 16, torch.float16)
    q = normal(g, 1, 3, 64, dtype=torch.float16)
    want = attend(c, q, table, lens)
    c.v[table[0, 1], 0, 3, 5] = float("inf")
    out, lse = torch.empty_like(q), torch.empty((1, 3), device="cuda")
    c.attention(q, table, lens, out, scale=64 ** -0.5)
    keep = [d for d in range(64) if d != 5]
    assert (out[0, :, 5] == float("inf")).all() and torch.equal(out[0][:, keep], want[0][:, keep])
    q.abs_().add_(1.0)
    c.k.fill_(0.0)
    c.k[..., 0] = float("-inf")
    c.v.fill_(60000.0)
    c.attention(q, table, lens, out, scale=64 ** -0.5, lse=lse)
    assert (out == 0).all() and (lse == float("-inf")).all()
    c.k[table[0, 2], 0, 0, 0] = 1.0
    c.v[table[0, 2], 0, 0] = 2.0 ** -14
    c.attention(q, table, lens, out, scale=64 ** -0.5, lse=lse)
    assert (out == 2.0 ** -14).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("scale", [0.125, 3.0, 1e3])          # weights that are all there, that fade, that are 0
@pytest.mark.parametrize("length", [40, 700, 20000])
def test_negative_scales(length, scale, dtype):
    """An 8-bit cache whose scales have either sign, or are 0: they multiply, whatever the weight."""
    g = gen(93)
    c, table, lens = build(g, [length, 3], 2, 64, 16, dtype, F8)
    for s in (c.k_scale, c.v_scale):
        s.mul_(torch.randint(-1, 2, s.shape, generator=g, device="cuda"))
    attend(c, normal(g, 2, 4, 64, dtype=dtype, std=2.0), table, lens, scale=scale)


@pytest.mark.parametrize("dtype,cache", [(torch.float16, None), (torch.bfloat16, F8)])
@pytest.mark.parametrize("dim,bound", [(112, 200), (120, 200), (120, 380), (128, 200), (232, 500), (240, 500), (248, 500), (256, 500)])
def test_workgroups_around_64_kib_of_lds(dim, bound, dtype, cache):
    """16 query heads to a key-value head, whole sequences by 8 waves (to 128) and chunks by 4: the sums and what the
    kernel holds beside them come to 60 to 70 KiB."""
    g = gen(dim)
    c, table, lens = build(g, [bound, 1, 77], 2, dim, 20, dtype, cache)
    assert (c.workspace_bytes(32, 3, bound) == 0) == (dim <= 128)
    attend(c, normal(g, 3, 32, dim, dtype=dtype, std=2.0), table, lens, max_length=bound)


def test_more_workgroups_than_fit_along_one_dimension():
    """65535 sequences under a bound of 33 chunks, 8 heads that share lines: 2^32 threads and more, most without a
    position."""
    n, kv, dim, page = 65535, 8, 8, 32768
    g = gen(94)
    c = A.KVCache(normal(g, 6, page, kv, dim, dtype=torch.float16), normal(g, 6, page, kv, dim, dtype=torch.float16), layout="slot")
    lens = torch.zeros((n,), dtype=torch.int32, device="cuda")
    table = torch.full((n, 5), -1, dtype=torch.int32, device="cuda")
    held = [0, 1, 4095, 40000, n - 1]
    for i, length in zip(held, (5000, 1, 32769, 100, 9000)):
        lens[i] = length
        table[i] = torch.randperm(6, generator=g, device="cuda")[:5]
    q = normal(g, n, kv, dim, dtype=torch.float16)
    out = torch.full_like(q, 9.0)
    bound = 33 * 4096
    assert n * 33 * kv * 256 >= 2 ** 32 and c.workspace_bytes(kv, n, bound) == n * kv * 33 * (dim + 2) * 4
    c.attention(q, table, lens, out, scale=0.3, max_length=bound)
    check(c, q[held], table[held], lens[held], 0.3, 0, out[held], None)
    out[held] = 0
    assert (out == 0).all()


@pytest.mark.parametrize("dtype,cache", [(torch.float16, None), (torch.bfloat16, F8)])
@pytest.mark.parametrize("layout,dim", [("head", 128), ("slot", 80)])
@pytest.mark.parametrize("bound,window", [(300, 0), (1300, 0), (1300, 1000), (20000, 0)])        # whole, few chunks, many
def test_neighbours_do_not_change_a_bit(bound, window, layout, dim, dtype, cache):
    """The same call but for the other sequences' lengths and pages: the same bits."""
    g = gen(95)
    lens_ = [bound, 7, bound // 2 + 1, bound - 1]
    c, table, lens = build(g, lens_, 2, dim, 16, dtype, cache, layout)
    q = normal(g, 4, 6, dim, dtype=dtype, std=2.0)

    def run(table, lens):
        out, lse = torch.empty_like(q), torch.empty((4, 6), device="cuda")
        c.attention(q, table, lens, out, scale=dim ** -0.5, max_length=bound, window=window, lse=lse)
        return out, lse

    want = run(table, lens)
    for keep in range(4):
        for other in (0, 1, bound // 3, bound):
            lens2, table2 = torch.full_like(lens, other), table[[3, 3, 3, 3]].clone()
            lens2[keep], table2[keep] = lens[keep], table[keep]
            got = run(table2, lens2)
            assert torch.equal(got[0][keep], want[0][keep]) and torch.equal(got[1][keep], want[1][keep])
