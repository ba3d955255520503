"""The operators' calls past ctypes: taken for the usual arguments, with the results of the other way, and left
alone for all else. (A stream given by the caller goes by ctypes.)"""
import pytest
import torch

A = pytest.importorskip("paper_2606_12876_amd", reason="libaqmb.so not built")
from paper_2606_12876_amd import _direct  # noqa: E402

BAD = [None, 1, "x", [], torch.zeros(2, 3), torch.zeros(0)]


def test_leaves_what_it_does_not_know():
    t = torch.zeros(2, 8, dtype=torch.float16)
    for n in (0, 1, 3, 5, 7, 9, 11):
        for f in (_direct.rms_norm, _direct.w4_gemv, _direct.paged_attention, _direct.kv_append, _direct.kv_copy_pages):
            for bad in BAD + [t]:
                assert f(*([bad] * n)) is None
    with pytest.raises(TypeError):
        _direct.bind(1, 2)
    with pytest.raises(ValueError):
        _direct.bind(0, 0, 0, 0, 0, 0)


def normal(*shape, dtype=torch.bfloat16):
    return torch.randn(*shape, device="cuda").to(dtype)


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("strided", [False, True])
def test_norm(strided, out):
    rows, cols = 5, 264
    wide = normal(3, rows, 2 * cols)
    x, r, r2 = (w[:, :cols] if strided else w[:, :cols].contiguous() for w in wide)
    w = torch.nn.Parameter(normal(cols), requires_grad=False)
    q8 = out in (torch.float8_e4m3fn, torch.int8)
    got = []
    for stream in (None, torch.cuda.current_stream()):
        y, sc = torch.zeros(rows, cols, dtype=out, device="cuda"), torch.zeros(rows, 3, device="cuda") if q8 else None
        ro = torch.zeros_like(wide[2])[:, :cols] if strided else torch.zeros_like(r2)
        a = (x, w, y, 1e-5, 0.5, r, ro, sc, 128 if q8 else 0)
        if stream is None:
            assert _direct.rms_norm(*a) == 0
        else:
            A.rms_norm(x, w, y, eps=1e-5, weight_offset=0.5, residual=r, residual_out=ro, scales=sc,
                       scale_group=128 if q8 else 0, stream=stream)
        got.append([y, ro.contiguous()] + ([sc] if q8 else []))
    for a, b in zip(*got):
        assert same(a, b)
    y = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    for bad in ((x, w[:8], y), (x, w, y[:, :8]), (x.float(), w, y), (x.cpu(), w, y), (x, w.cpu(), y), (x[:0], w, y[:0]),
                (x.t(), w, y.t())):
        assert _direct.rms_norm(*bad, 1e-5, 0.0, None, None, None, 0) is None
        with pytest.raises(A.AqmbError):
            A.rms_norm(*bad, eps=1e-5)
    assert _direct.rms_norm(x, w, y, 1e-5, 0.0, r, None, None, 0) is None
    assert _direct.rms_norm(x, w, y, 1e-5, 0.0, None, None, torch.zeros(1, device="cuda"), 32) is None
    torch.cuda.synchronize()
    assert (y == 0).all()
    # the library's own refusal comes back as its status, and from the binding with its message
    z = torch.zeros(rows, cols, dtype=torch.int8, device="cuda")
    assert _direct.rms_norm(x, w, z, 1e-5, 0.0, None, None, None, 0) == A.Status.EINVAL
    with pytest.raises(A.AqmbError, match="scales"):
        A.rms_norm(x, w, z, eps=1e-5)


@pytest.mark.gpu
def test_w4():
    d_out, d_in, g = 80, 320, 64
    layer = A.W4Linear(torch.randint(0, 256, (d_out, d_in // 2), device="cuda").to(torch.uint8),
                       torch.rand(d_out, d_in // g, device="cuda").half(), group_size=g)
    for x, sx in ((normal(3, d_in), None), (normal(3, 2 * d_in)[:, d_in:], None),
                  (torch.randint(-99, 99, (3, d_in), device="cuda").to(torch.int8), torch.rand(3, 1, device="cuda")),
                  (normal(3, d_in).to(torch.float8_e4m3fn), torch.rand(3, d_in // g, device="cuda"))):
        y, z = (torch.zeros(3, d_out, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        assert _direct.w4_gemv(layer.handle, d_out, d_in, g, x, y, sx) == 0
        layer.gemv(x, z, sx, stream=torch.cuda.current_stream())
        assert same(y, z) and (y != 0).any()
    x, y = normal(3, d_in), torch.zeros(3, d_out, dtype=torch.bfloat16, device="cuda")
    for bad in ((None, d_out, d_in, g, x, y, None), (layer.handle, d_out, d_in, g, x[:, 1:], y, None),
                (layer.handle, d_out, d_in, g, x, y[:2], None), (layer.handle, d_out, d_in, g, x, y, x)):
        assert _direct.w4_gemv(*bad) is None
    assert _direct.w4_gemv(layer.handle, d_out, d_in, g, normal(17, d_in), normal(17, d_out), None) == A.Status.EUNSUPPORTED
    torch.cuda.synchronize()
    assert (y == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("per", [4, 90])
def test_attention_and_cache(per):
    """Without and with a workspace of the call's own."""
    n, heads, kv, dim, page = 3, 8, 2, 64, 16
    c = A.KVCache.allocate(4 * n * per, page, kv, dim, torch.bfloat16)
    c.k.normal_(), c.v.normal_()
    table = torch.randperm(c.n_pages, device="cuda")[:n * per].view(n, per).to(torch.int32)
    lens = torch.tensor([per * page, 0, 33], dtype=torch.int32, device="cuda")
    qkv = normal(n, heads + 2 * kv, dim)
    q = qkv[:, :heads]
    need = c.workspace_bytes(heads, n, per * page)
    assert (need > 0) == (per == 90)
    got = []
    for way in range(3):
        out, lse = torch.zeros(n, heads, dim, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, heads, device="cuda")
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if way == 1 else None
        if way < 2:
            assert _direct.paged_attention(c._address, c.device_index, q, table, lens, out, 0.125, None, 0, lse, ws) == 0
        else:
            c.attention(q, table, lens, out, scale=0.125, lse=lse, stream=torch.cuda.current_stream())
        got.append((out, lse))
    for other in got[1:]:
        assert same(got[0][0], other[0]) and same(got[0][1], other[1])
    out = torch.zeros_like(got[0][0])
    ok = [c._address, c.device_index, q, table, lens, out, 0.125, None, 0, None, None]
    for i, bad in ((0, 0), (1, c.device_index + 1), (2, q[:, :, :32]), (2, q.float()), (3, table.long()), (3, table[:2]),
                   (4, lens[:2]), (4, lens.float()), (5, out[:2]), (5, out.half()), (6, 1), (7, per * page + 1), (7, -1),
                   (8, -1), (9, lens), (10, "x")):
        args = list(ok)
        args[i] = bad
        assert _direct.paged_attention(*args) is None, i
    torch.cuda.synchronize()
    assert (out == 0).all()
    if need:
        assert _direct.paged_attention(*ok[:10], torch.empty(16, dtype=torch.uint8, device="cuda")) == A.Status.EINVAL

    k, v = qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    slots = torch.tensor([5, -1, 40], device="cuda")
    assert _direct.kv_append(c._address, c.device_index, k, v, slots) == 0
    at = table.new_zeros(0)
    assert same(c.k[0, :, 5].contiguous(), k[0].contiguous()) and same(c.v[2, :, 8].contiguous(), v[2].contiguous())
    for i, bad in ((0, 0), (2, k[:, :1]), (3, v.half()), (4, slots.int()), (4, slots[:2]), (4, at)):
        args = [c._address, c.device_index, k, v, slots]
        args[i] = bad
        assert _direct.kv_append(*args) is None

    other = A.KVCache.allocate(c.n_pages, page, kv, dim, torch.bfloat16)
    other.k.normal_(), other.v.normal_()
    src, dst = (torch.tensor(p, dtype=torch.int32, device="cuda") for p in ([1, 2], [5, 6]))
    assert _direct.kv_copy_pages([c, other], src, dst) == 0
    assert same(c.k[5:7], c.k[1:3]) and same(other.v[5:7], other.v[1:3])
    A.kv_copy_pages((x for x in (c, other)), dst, src + 6)
    assert same(c.v[7:9], c.v[5:7]) and same(other.k[7:9], other.k[5:7])
    for bad in (([], src, dst), ([c, 1], src, dst), ([c] * 65, src, dst), ([c], src, dst[:1]), ([c], src.long(), dst),
                (c, src, dst)):
        assert _direct.kv_copy_pages(*bad) is None


@pytest.mark.gpu
def test_current_stream():
    """The call goes to the stream that is current, its workspace with it."""
    s = torch.cuda.Stream()
    x, w = normal(4, 512), normal(512)
    y = torch.zeros_like(x)
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        assert _direct.rms_norm(x, w, y, 1e-5, 0.0, None, None, None, 0) == 0
    torch.cuda.synchronize()
    assert (y == 0).all()           # recorded, not run
    g.replay()
    torch.cuda.synchronize()
    z = torch.zeros_like(x)
    A.rms_norm(x, w, z, eps=1e-5)
    assert same(y, z) and (y != 0).any()
