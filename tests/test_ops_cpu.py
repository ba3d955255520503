"""The operators between the layers on the CPU: exports, refusals before any launch, page bookkeeping."""
import ctypes
import os
import random
import re

import pytest

A = pytest.importorskip("paper_2606_12876_amd", reason="libaqmb.so not built")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
S = A.Status
F16, BF16, F32, F8, I8 = 0, 1, 2, 3, 4


def test_exports_every_declared_symbol_with_digits_too():
    hdr = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "aqmb.h")).read(), flags=re.S)
    syms = set(re.findall(r"\b(aqmb_[a-z0-9_]+)\s*\(", hdr))
    assert {"aqmb_rms_norm", "aqmb_w4_gemv", "aqmb_paged_attention", "aqmb_kv_append", "aqmb_pages_extend"} <= syms
    for s in syms:
        assert hasattr(A.lib, s), s


def norm(**kw):
    a = dict(x=16, dtype=BF16, xs=64, r=None, ro=None, rs=0, w=16, w0=0.0, eps=1e-6, rows=2, cols=64, y=16, yd=BF16,
             ys=64, sc=None, g=0)
    a.update(kw)
    return A.lib.aqmb_rms_norm(a["x"], a["dtype"], a["xs"], a["r"], a["ro"], a["rs"], a["w"], a["w0"], a["eps"],
                               a["rows"], a["cols"], a["y"], a["yd"], a["ys"], a["sc"], a["g"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=F32), S.EUNSUPPORTED), (dict(dtype=F8), S.EUNSUPPORTED), (dict(yd=9), S.EUNSUPPORTED),
    (dict(x=None), S.EINVAL), (dict(w=None), S.EINVAL), (dict(y=None), S.EINVAL),
    (dict(r=16), S.EINVAL), (dict(ro=16), S.EINVAL), (dict(r=16, ro=16, rs=63), S.EINVAL),
    (dict(rows=0), S.EINVAL), (dict(cols=0), S.EINVAL), (dict(cols=32769, xs=32769, ys=32769), S.EUNSUPPORTED),
    (dict(xs=63), S.EINVAL), (dict(ys=63), S.EINVAL),
    (dict(eps=-1e-6), S.EINVAL), (dict(eps=float("nan")), S.EINVAL), (dict(eps=float("inf")), S.EINVAL),
    (dict(yd=F8), S.EINVAL), (dict(sc=16), S.EINVAL), (dict(yd=I8, sc=16, g=48), S.EUNSUPPORTED),
    (dict(yd=I8, sc=16, g=-32), S.EUNSUPPORTED), (dict(yd=I8, sc=18), S.EINVAL),
    (dict(x=17), S.EINVAL), (dict(w=17), S.EINVAL), (dict(y=18, yd=F32), S.EINVAL), (dict(r=17, ro=16, rs=64), S.EINVAL),
])
def test_rms_norm_refuses(kw, status):
    assert norm(**kw) == status
    assert A.last_error()


@pytest.mark.parametrize("d_out,d_in,g,w,s,status", [
    (0, 64, 32, 16, 16, S.EINVAL), (4, 0, 32, 16, 16, S.EINVAL), (4, 64, 16, 16, 16, S.EUNSUPPORTED),
    (4, 64, 256, 16, 16, S.EUNSUPPORTED), (1 << 17, 1 << 15, 32, 16, 16, S.EINVAL),
    (1, (1 << 30) + 1, 32, 16, 16, S.EINVAL), ((1 << 30) + 1, 1, 32, 16, 16, S.EINVAL), (4, 64, 32, None, 16, S.EINVAL),
    (4, 64, 32, 16, None, S.EINVAL), (4, 64, 32, 16, 17, S.EINVAL)])
def test_w4_create_refuses(d_out, d_in, g, w, s, status):
    h, d = ctypes.c_void_p(0x1234), A.W4Desc(d_out, d_in, g)
    assert A.lib.aqmb_w4_create(ctypes.byref(h), ctypes.byref(d), w, s, None, None) == status
    assert h.value is None and A.last_error()


def test_w4_handles():
    bogus = ctypes.c_void_p(0x1000)
    assert A.lib.aqmb_w4_create(None, None, 16, 16, None, None) == S.EINVAL
    assert A.lib.aqmb_w4_destroy(None) == S.OK
    assert A.lib.aqmb_w4_destroy(bogus) == S.EINVAL
    assert A.lib.aqmb_w4_get_desc(bogus, None) == S.EINVAL
    assert A.lib.aqmb_w4_gemv(bogus, 16, F16, 64, None, 0, 1, 16, F16, 64, None) == S.EINVAL
    assert "live" in A.last_error()


def cache(**kw):
    a = dict(k=64, v=64, k_scale=None, v_scale=None, page_stride=2 * 16 * 64, dtype=BF16, layout=0, n_pages=4,
             page_size=16, n_kv_heads=2, head_dim=64)
    a.update(kw)
    return A.KVCacheDesc(*[a[n] for n, _ in A.KVCacheDesc._fields_])


BAD_CACHES = [
    (dict(dtype=F32), S.EUNSUPPORTED), (dict(dtype=I8), S.EUNSUPPORTED), (dict(layout=2), S.EINVAL),
    (dict(n_pages=0), S.EINVAL), (dict(page_size=0), S.EINVAL), (dict(n_kv_heads=0), S.EINVAL), (dict(head_dim=0), S.EINVAL),
    (dict(page_size=32769), S.EUNSUPPORTED), (dict(head_dim=60), S.EUNSUPPORTED),
    (dict(head_dim=264, page_stride=1 << 20), S.EUNSUPPORTED), (dict(page_stride=2040), S.EINVAL),
    (dict(page_stride=2052), S.EINVAL), (dict(k=None), S.EINVAL), (dict(v=None), S.EINVAL), (dict(k=72), S.EINVAL),
    (dict(dtype=F8), S.EINVAL), (dict(dtype=F8, k_scale=64), S.EINVAL), (dict(dtype=F8, k_scale=64, v_scale=66), S.EINVAL),
    (dict(k_scale=64, v_scale=64), S.EINVAL)]


def attend(c, **kw):
    a = dict(q=64, dtype=BF16, qs=256, heads=4, table=64, ts=4, lens=64, n=2, ml=64, scale=1.0, window=0, out=64, os=256,
             lse=None, ws=None, wb=0)
    a.update(kw)
    return A.lib.aqmb_paged_attention(ctypes.byref(c) if c else None, a["q"], a["dtype"], a["qs"], a["heads"], a["table"],
                                      a["ts"], a["lens"], a["n"], a["ml"], a["scale"], a["window"], a["out"], a["os"],
                                      a["lse"], a["ws"], a["wb"], None)


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_every_cache_call_refuses_a_bad_cache(kw, status):
    c = cache(**kw)
    n = ctypes.c_size_t(7)
    assert attend(c) == status
    assert A.lib.aqmb_paged_attention_workspace_bytes(ctypes.byref(c), 4, 2, 64, 0, ctypes.byref(n)) == status
    assert A.lib.aqmb_kv_append(ctypes.byref(c), 64, 128, 64, 128, BF16, 64, 3, None) == status
    assert A.lib.aqmb_kv_copy_pages((A.KVCacheDesc * 1)(c), 1, 64, 64, 2, None) == status
    assert A.last_error() and n.value == 7


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=F16), S.EUNSUPPORTED), (dict(dtype=F32), S.EUNSUPPORTED), (dict(heads=3), S.EINVAL), (dict(heads=0), S.EINVAL),
    (dict(n=0), S.EINVAL), (dict(n=65536), S.EUNSUPPORTED), (dict(ml=-1), S.EINVAL), (dict(ml=65), S.EINVAL),
    (dict(ml=(1 << 30) + 1, ts=1 << 40), S.EINVAL), (dict(window=-1), S.EINVAL), (dict(q=None), S.EINVAL),
    (dict(table=None), S.EINVAL), (dict(lens=None), S.EINVAL), (dict(out=None), S.EINVAL), (dict(qs=248), S.EINVAL),
    (dict(os=260), S.EINVAL), (dict(q=72), S.EINVAL), (dict(out=72), S.EINVAL), (dict(lens=66), S.EINVAL),
    (dict(lse=66), S.EINVAL), (dict(ts=0), S.EINVAL), (dict(scale=float("inf")), S.EINVAL),
    (dict(scale=float("nan")), S.EINVAL)])
def test_attention_refuses(kw, status):
    assert attend(cache(), **kw) == status
    assert A.last_error()


def test_calls_past_one_launch_are_refused():
    c = cache(n_kv_heads=8, page_stride=1 << 20)
    assert A.lib.aqmb_kv_append(ctypes.byref(c), 64, 1 << 12, 64, 1 << 12, BF16, 64, 1 << 23, None) == S.EUNSUPPORTED
    assert "2^26" in A.last_error()
    for rows, cols in ((1 << 22, 4096), (1 << 27, 128), (1 << 28, 64), (2 ** 31 - 1, 1), (1 << 19, 32768)):
        assert A.lib.aqmb_rms_norm(64, BF16, cols, None, None, 0, 64, 0.0, 1e-5, rows, cols, 64, BF16, cols, None, 0,
                                   None) == S.EUNSUPPORTED
        assert "one launch" in A.last_error()


def test_append_and_copy_refuse():
    c = cache()
    f = A.lib.aqmb_kv_append
    ref = ctypes.byref(c)
    assert f(None, 64, 128, 64, 128, BF16, 64, 3, None) == S.EINVAL
    assert f(ref, None, 128, 64, 128, BF16, 64, 3, None) == S.EINVAL
    assert f(ref, 64, 128, 64, 128, BF16, None, 3, None) == S.EINVAL
    assert f(ref, 64, 127, 64, 128, BF16, 64, 3, None) == S.EINVAL
    assert f(ref, 64, 128, 64, 127, BF16, 64, 3, None) == S.EINVAL
    assert f(ref, 64, 128, 64, 128, BF16, 64, 0, None) == S.EINVAL
    assert f(ref, 65, 128, 64, 128, BF16, 64, 3, None) == S.EINVAL
    assert f(ref, 64, 128, 64, 128, BF16, 68, 3, None) == S.EINVAL
    assert f(ref, 64, 128, 64, 128, F16, 64, 3, None) == S.EUNSUPPORTED
    two = (A.KVCacheDesc * 2)(c, cache(n_pages=5))
    g = A.lib.aqmb_kv_copy_pages
    assert g(two, 2, 64, 64, 1, None) == S.EINVAL and "differs" in A.last_error()
    assert g(None, 1, 64, 64, 1, None) == S.EINVAL
    assert g(two, 0, 64, 64, 1, None) == S.EINVAL
    assert g(two, 1, 64, 64, 0, None) == S.EINVAL
    assert g(two, 1, None, 64, 1, None) == S.EINVAL
    assert g((A.KVCacheDesc * 65)(*[cache() for _ in range(65)]), 65, 64, 64, 1, None) == S.EUNSUPPORTED


# -------------------------------------------------------------------------------- page bookkeeping
class Model:
    """What the pool promises, the slow way: every token of every sequence has a value, pages hold them."""

    def __init__(self, n_pages, size):
        self.pages = [[None] * size for _ in range(n_pages)]
        self.size, self.text = size, {}

    def write(self, slots, values, copies):
        for s, d in copies:
            self.pages[d] = list(self.pages[s])
        for slot, v in zip(slots, values):
            self.pages[slot // self.size][slot % self.size] = v

    def check(self, pool):
        holders = {}
        for seq, text in self.text.items():
            table = pool.table(seq).tolist()
            assert pool.length(seq) == len(text)
            assert len(table) == -(-len(text) // self.size) and len(set(table)) == len(table)
            assert [self.pages[table[t // self.size]][t % self.size] for t in range(len(text))] == text
            for p in table:
                holders[p] = holders.get(p, 0) + 1
        free, live = pool.counts()
        assert live == len(self.text) and free == len(self.pages) - len(holders)
        return set(holders)


@pytest.mark.parametrize("seed", range(12))
def test_page_pool_against_a_model(seed):
    rng = random.Random(seed)
    n_pages, size, seqs = rng.choice([(1, 1, 1), (7, 4, 3), (40, 1, 9), (33, 16, 8), (64, 5, 20)])
    pool, model, stamp = A.PagePool(n_pages, size, seqs), Model(n_pages, size), 0
    for _ in range(300):
        op = rng.choice(["add", "extend", "extend", "extend", "fork", "free", "compact"])
        some = rng.choice(sorted(model.text)) if model.text else None
        if op == "add" or (op == "fork" and some is not None):
            if len(model.text) == seqs:
                with pytest.raises(A.AqmbError) as e:
                    pool.add() if op == "add" else pool.fork(some)
                assert e.value.status == S.ENOMEM
            else:
                new = pool.add() if op == "add" else pool.fork(some)
                assert new == min(set(range(seqs)) - set(model.text))
                model.text[new] = [] if op == "add" else list(model.text[some])
        elif op == "extend" and some is not None:
            n = rng.choice([0, 1, 1, size - 1, size, rng.randint(0, 3 * size)])
            before = pool.table(some).tolist()
            others = {p for t in model.text if t != some for p in pool.table(t).tolist()}
            at = len(model.text[some])
            shared = n > 0 and at % size != 0 and before[-1] in others
            fresh = -(-(at + n) // size) - len(before) + shared
            if fresh > pool.counts()[0]:
                with pytest.raises(A.AqmbError) as e:
                    pool.extend(some, n)
                assert e.value.status == S.ENOMEM and pool.table(some).tolist() == before
            else:
                slots, copies = pool.extend(some, n)
                assert len(slots) == n and bool(copies) == shared
                values = list(range(stamp, stamp + n))
                stamp += n
                model.write(slots.tolist(), values, copies)
                model.text[some] += values
        elif op == "free" and some is not None:
            pool.free(some)
            del model.text[some]
        elif op == "compact":
            pairs = pool.compact()
            src, dst = [p[0] for p in pairs], [p[1] for p in pairs]
            assert len(set(dst)) == len(dst) and not set(src) & set(dst)
            for s, d in pairs:
                model.pages[d] = list(model.pages[s])
            used = model.check(pool)
            assert used == set(range(len(used)))
        model.check(pool)
    pool.close()


def test_page_pool_refuses():
    for bad in ((0, 4, 4), (4, 0, 4), (4, 4, 0)):
        with pytest.raises(A.AqmbError) as e:
            A.PagePool(*bad)
        assert e.value.status == S.EINVAL
    bogus, i = ctypes.c_void_p(0x1000), ctypes.c_int(-7)
    assert A.lib.aqmb_pages_destroy(None) == S.OK
    assert A.lib.aqmb_pages_destroy(bogus) == S.EINVAL
    assert A.lib.aqmb_pages_add(bogus, ctypes.byref(i)) == S.EINVAL and i.value == -7
    pool = A.PagePool(4, 4, 2)
    s = pool.add()
    for f in (lambda: pool.free(1), lambda: pool.free(-1), lambda: pool.free(2), lambda: pool.fork(1),
              lambda: pool.extend(1, 1), lambda: pool.extend(s, -1), lambda: pool.table(1), lambda: pool.length(5)):
        with pytest.raises(A.AqmbError) as e:
            f()
        assert e.value.status == S.EINVAL
    n, length, src = ctypes.c_int(), ctypes.c_int(), ctypes.c_int32()
    assert A.lib.aqmb_pages_extend(pool.handle, s, 3, None, ctypes.byref(src), ctypes.byref(src)) == S.EINVAL
    assert A.lib.aqmb_pages_extend(pool.handle, s, 0, None, None, ctypes.byref(src)) == S.EINVAL
    pool.extend(s, 5)
    small = (ctypes.c_int32 * 1)()
    assert A.lib.aqmb_pages_table(pool.handle, s, small, 1, ctypes.byref(n), ctypes.byref(length)) == S.EINVAL
    assert (n.value, length.value) == (2, 5)
    assert A.lib.aqmb_pages_compact(pool.handle, None, None, ctypes.byref(n)) == S.EINVAL
    pool.extend(s, 11)
    with pytest.raises(A.AqmbError) as e:
        pool.extend(s, 1)
    assert e.value.status == S.ENOMEM
    pool.close()
    assert A.lib.aqmb_pages_add(bogus, ctypes.byref(i)) == S.EINVAL


@pytest.mark.parametrize("d_out,d_in", [(1 << 28, 1), (1 << 30, 3), ((1 << 28) - 15, 15), (1 << 21, 2000), (1, 1 << 30)])
def test_w4_create_refuses_what_one_launch_cannot_lay_out(d_out, d_in):
    """Tall, narrow layers are mostly padding: a thread for every dword of the tiles, fewer than 2^32."""
    fits = -(-d_out // 16) * -(-d_in // 128) < 1 << 24
    h, d = ctypes.c_void_p(0x1234), A.W4Desc(d_out, d_in, 128)
    if fits:        # refused for something that is looked at later
        assert A.lib.aqmb_w4_create(ctypes.byref(h), ctypes.byref(d), None, 16, None, None) == S.EINVAL
        assert "NULL" in A.last_error()
    else:
        assert A.lib.aqmb_w4_create(ctypes.byref(h), ctypes.byref(d), 16, 16, None, None) == S.EINVAL
        assert "tiles" in A.last_error()
    assert h.value is None


def test_launches_are_counted_in_whole_workgroups():
    """One row, or one token's head, below the limits still rounds up to a launch of 2^32 threads."""
    c = cache(n_kv_heads=1, page_stride=1 << 20)
    for tokens in ((1 << 26) - 3, (1 << 26) - 1):
        assert A.lib.aqmb_kv_append(ctypes.byref(c), 64, 64, 64, 64, BF16, 64, tokens, None) == S.EUNSUPPORTED
        assert "2^26" in A.last_error()
    for rows in ((1 << 28) - 15, (1 << 28) - 1):
        for cols in (1, 64):
            assert A.lib.aqmb_rms_norm(64, BF16, cols, None, None, 0, 64, 0.0, 1e-5, rows, cols, 64, BF16, cols, None, 0,
                                       None) == S.EUNSUPPORTED
            assert "one launch" in A.last_error()
