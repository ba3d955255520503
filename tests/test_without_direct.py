"""The package without _direct.so: it imports, with a warning, and every call reaches the same kernels through ctypes;
the build yields the libraries whatever becomes of it."""
import importlib.util
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = pytest.importorskip("paper_2606_12876_amd", reason="libaqmb.so not built")


def test_the_package_imports_without_it():
    code = """
import sys, warnings
class Block:
    def find_spec(self, name, path=None, target=None):
        if name == "paper_2606_12876_amd._direct":
            raise ImportError("undefined symbol")
sys.meta_path.insert(0, Block())
with warnings.catch_warnings(record=True) as seen:
    warnings.simplefilter("always")
    import paper_2606_12876_amd as A
assert A._direct is None and any("_direct.so" in str(w.message) for w in seen), seen
pool = A.PagePool(4, 4, 2)
assert len(pool.extend(pool.add(), 3)[0]) == 3
assert A.validate and A.QuantLinear and A.W4Linear and A.KVCache
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def load_build():
    spec = importlib.util.spec_from_file_location("build_under_test", os.path.join(ROOT, "paper_2606_12876_amd", "build.py"))
    b = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(b)
    return b


@pytest.mark.parametrize("case", ["all there", "no headers", "no torch", "does not compile"])
def test_the_libraries_are_built_first(case, monkeypatch, tmp_path):
    b = load_build()
    linked, compiled = [], []

    def compile_(src):
        compiled.append(src)
        if src in b.DIRECT_SOURCES and case == "does not compile":
            raise RuntimeError("compiling direct.cpp failed")
        return src

    monkeypatch.setattr(b, "_compile", compile_)
    monkeypatch.setattr(b, "_link", lambda objs, lib, more=(): linked.append(lib))
    monkeypatch.setattr(b, "BUILD", str(tmp_path))
    monkeypatch.setattr(b, "DIRECT_LIB", str(tmp_path / "_direct.so"))
    (tmp_path / "_direct.so").write_text("old")
    if case == "no headers":
        monkeypatch.setattr(b.sysconfig, "get_paths", lambda: {"include": str(tmp_path / "nowhere")})
    if case == "no torch":
        monkeypatch.setattr(b.importlib.util, "find_spec", lambda name: None)
    if case == "does not compile":
        with pytest.raises(RuntimeError, match="direct.cpp"):
            b.build()
    else:
        assert b.build() == b.LIB
    assert linked == [b.LIB, b.CEIL_LIB] + ([b.DIRECT_LIB] if case == "all there" else [])
    assert (b.DIRECT_SOURCES[0] in compiled) == (case in ("all there", "does not compile"))
    assert not (tmp_path / "_direct.so").exists()


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")
def test_the_same_results(monkeypatch):
    g = torch.Generator(device="cuda")
    g.manual_seed(1)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)

    x, r, w = normal(5, 264), normal(5, 264), normal(264)
    layer = A.W4Linear(torch.randint(0, 256, (80, 132), generator=g, device="cuda").to(torch.uint8),
                       torch.rand((80, 5), generator=g, device="cuda").half(), group_size=64)
    new, q = normal(3, 2, 64), normal(3, 8, 64)
    stored = normal(2, 300, 2, 16, 64)
    table = torch.randperm(300, generator=g, device="cuda")[:270].view(3, 90).to(torch.int32)
    lens = torch.tensor([1440, 0, 33], dtype=torch.int32, device="cuda")
    slots = torch.tensor([5, -1, 40], device="cuda")
    src, dst = (torch.tensor(p, dtype=torch.int32, device="cuda") for p in ([1, 2], [5, 6]))

    def everything():
        y8, sc, r2 = torch.empty((5, 264), dtype=torch.int8, device="cuda"), torch.empty((5, 5), device="cuda"), torch.empty_like(x)
        A.rms_norm(x, w, y8, eps=1e-5, residual=r, residual_out=r2, scales=sc, scale_group=64)
        c = A.KVCache(*(t.clone() for t in stored))
        assert c.workspace_bytes(8, 3, 1440) > 0
        c.append(new, -new, slots)
        A.kv_copy_pages([c], src, dst)
        out, lse = torch.empty_like(q), torch.empty((3, 8), device="cuda")
        c.attention(q, table, lens, out, scale=0.125, lse=lse)
        return y8, sc, r2, layer(y8, sc), c.k, c.v, out, lse

    want = everything()
    monkeypatch.setattr(A, "_direct", None)
    for a, b in zip(want, everything()):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    with pytest.raises(A.AqmbError, match="dense"):
        A.rms_norm(x, w[::2], y=torch.empty_like(x), eps=1e-5)
    layer.close()
