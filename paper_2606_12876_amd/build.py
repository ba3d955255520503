"""Compile libaqmb.so for gfx950 in-tree (hipcc cross-compiles; no GPU needed).

Objects go to ``_build/`` at the repository root; the shared library is written next to
this file, where the binding loads it. Every HIP source is compiled with packed-fp32
instruction generation turned off. ``libaqmb_ceilings.so`` (the benchmark's measured-ceiling
kernels, not part of the layer) and ``_direct.so`` (the binding's way from tensors to the library
without ctypes; host code against the headers of Python and of the installed PyTorch, left out where those
are missing) are built beside it.
"""
from __future__ import annotations

import concurrent.futures as cf
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libaqmb.so")
CEIL_SOURCES = ["ceilings.hip"]
DIRECT_SOURCES = ["direct.cpp"]
CEIL_LIB = os.path.join(HERE, "libaqmb_ceilings.so")
DIRECT_LIB = os.path.join(HERE, "_direct.so")

SOURCES = ["validate.cpp", "api.cpp", "k_dequant.hip", "k_gemv.hip", "k_gemv16.hip", "k_gemv4.hip", "k_gemv_mma.hip", "k_gemm.hip", "k_gemm_small.hip", "k_gemm_mid.hip", "k_distortion.hip", "k_beam.hip", "k_beam_mma.hip", "ops_api.cpp", "pages.cpp",
           "k_norm.hip", "k_w4.hip", "k_attn.hip", "k_kv.hip", "k_rotary.hip", "k_adapters.hip", "k_logprobs.hip"]
ARCH = "gfx950"


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found: install ROCm or set HIPCC")


def _flags(src: str):
    common = ["-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function", f"-I{os.path.join(ROOT, 'include')}"]
    if src.endswith(".hip"):
        return ["-x", "hip", f"--offload-arch={ARCH}", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"] + common
    if src in DIRECT_SOURCES:
        inc = [sysconfig.get_paths()["include"], os.path.join(_torch(), "include"), os.path.join(_rocm(), "include")]
        return common + ["-fvisibility=hidden", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1"] + \
            [a for i in inc for a in ("-isystem", i)]
    return common


def _rocm() -> str:
    return os.path.dirname(os.path.dirname(os.path.realpath(hipcc())))


def _torch() -> str:
    """The installed PyTorch's folder (found, not imported: it would load its HIP runtime), "" if there is none."""
    spec = importlib.util.find_spec("torch")
    return os.path.dirname(spec.origin) if spec and spec.origin else ""


def _direct_lacks() -> str:
    """The header that ``_direct.so`` needs and this machine does not have, "" if all are there."""
    for header in (os.path.join(sysconfig.get_paths()["include"], "Python.h"),
                   os.path.join(_torch(), "include", "torch", "csrc", "autograd", "python_variable.h"),
                   os.path.join(_rocm(), "include", "hip", "hip_runtime_api.h")):
        if not os.path.exists(header):
            return header
    return ""


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [hipcc()] + _flags(src) + ["-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compiling {src} failed:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def _link(objs, lib, more=()):
    tmp = lib + ".tmp"
    cmd = [hipcc(), "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp] + objs + list(more)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"linking failed:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, lib)


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    missing = _direct_lacks()
    srcs = SOURCES + CEIL_SOURCES + ([] if missing else DIRECT_SOURCES)
    jobs = min(len(srcs), max(1, min(16, os.cpu_count() or 1)))
    with cf.ThreadPoolExecutor(jobs) as ex:
        objs = {s: ex.submit(_compile, s) for s in srcs}
    _link([objs[s].result() for s in SOURCES], LIB)
    _link([objs[s].result() for s in CEIL_SOURCES], CEIL_LIB)
    # The libraries are there; _direct.so, which the binding can do without, comes last. An old one must not stay.
    if os.path.exists(DIRECT_LIB):
        os.remove(DIRECT_LIB)
    if missing:
        print(f"{DIRECT_LIB} is not built: {missing} not found", file=sys.stderr)
    else:
        # PyTorch's libraries are found by name: the package imports torch first.
        _link([objs[s].result() for s in DIRECT_SOURCES], DIRECT_LIB,
              ["-L" + os.path.join(_torch(), "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip"])
    if verbose:
        print(f"built {LIB}, {CEIL_LIB}" + ("" if missing else f" and {DIRECT_LIB}"))
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
