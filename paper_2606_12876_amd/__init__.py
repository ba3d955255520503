"""aqmb: multi-bitwidth additive-codebook linear layers on MI355X (gfx950).

Thin ctypes binding over ``libaqmb.so`` (``include/aqmb.h``). The functions here have the
C names without the ``aqmb_`` prefix and only marshal arguments: every step of the
computation runs in the library's HIP kernels. PyTorch tensors are accepted for device
buffers and the current PyTorch stream is used when no stream is given; PyTorch is plumbing
(allocation and streams), not part of the computation.

If the library has not been built, importing this package fails loudly: there is no
fallback implementation. ``_direct.so``, which takes usual calls past ctypes, may be missing:
a warning says so, and every call reaches the same kernels through ctypes.
"""
from __future__ import annotations

import ctypes
import enum
import os
import warnings
from typing import Optional

__all__ = ["Status", "DType", "Desc", "AqmbError", "GemvKernel", "GemmTiling", "lib", "create", "destroy", "get_desc",
           "gemv", "gemv_select", "gemm", "gemm_select", "dequant", "bits_per_weight", "strerror", "last_error",
           "validate", "QuantLinear", "LIB_PATH", "KVLayout", "W4Desc", "rms_norm", "w4_create", "w4_destroy",
           "w4_get_desc", "w4_gemv", "W4Linear", "KVCache", "paged_attention", "paged_attention_workspace_bytes",
           "kv_append", "kv_copy_pages", "PagePool"]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libaqmb.so")


class Status(enum.IntEnum):
    OK = 0
    EINVAL = 1
    EUNSUPPORTED = 2
    ENOMEM = 3
    EHIP = 4


class DType(enum.IntEnum):
    F16 = 0
    BF16 = 1
    F32 = 2
    F8 = 3       # e4m3; only the operators between the layers take it, with scales
    I8 = 4


class KVLayout(enum.IntEnum):
    """aqmb_kv_layout: the order inside a page of a key-value cache."""
    HEAD_MAJOR = 0
    SLOT_MAJOR = 1


class GemvKernel(enum.IntEnum):
    """aqmb_gemv_kernel: which GEMV kernel aqmb_gemv_select runs."""
    AUTO = 0
    DIRECT = 1
    MMA = 2
    LUT = 3


class GemmTiling(enum.IntEnum):
    """aqmb_gemm_tiling: which tiling aqmb_gemm_select runs."""
    AUTO = 0
    ROWS16 = 1
    T256x128 = 2
    T128x128 = 3
    T128x64 = 4


class Desc(ctypes.Structure):
    _fields_ = [("d_out", ctypes.c_int32), ("d_in", ctypes.c_int32), ("group_size", ctypes.c_int32),
                ("num_codebooks", ctypes.c_int32), ("code_bits", ctypes.c_int32)]


class W4Desc(ctypes.Structure):
    _fields_ = [("d_out", ctypes.c_int32), ("d_in", ctypes.c_int32), ("group_size", ctypes.c_int32)]


class KVCacheDesc(ctypes.Structure):
    """aqmb_kv_cache."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("page_stride", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("layout", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


class AqmbError(RuntimeError):
    def __init__(self, status: int, where: str, message: str):
        self.status = Status(status)
        super().__init__(f"{where}: {self.status.name}: {message}")


def _load() -> ctypes.CDLL:
    # One HIP runtime per process: PyTorch ships its own libamdhip64 (same SONAME). Importing
    # torch first makes the library bind to that runtime, so device pointers, streams and
    # devices are shared; loading the library first would start a second runtime.
    import torch  # noqa: F401
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it first (python -m paper_2606_12876_amd.build "
                          f"or __graft_entry__.build()); there is no fallback implementation")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, st = ctypes.c_void_p, ctypes.c_int, ctypes.c_int
    L.aqmb_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(Desc), vp, vp, vp, vp]
    L.aqmb_destroy.argtypes = [vp]
    L.aqmb_create_prefix.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(Desc), i32, vp, vp, vp, vp]
    L.aqmb_load_planes.argtypes = [vp, i32, vp, vp]
    L.aqmb_drop_planes.argtypes = [vp, i32]
    L.aqmb_resident_planes.argtypes = [vp, ctypes.POINTER(i32)]
    L.aqmb_get_desc.argtypes = [vp, ctypes.POINTER(Desc)]
    L.aqmb_gemv.argtypes = [vp, i32, vp, i32, i32, vp, i32, vp]
    L.aqmb_gemv_select.argtypes = [vp, i32, vp, i32, i32, vp, i32, i32, vp]
    L.aqmb_gemm_select.argtypes = [vp, i32, vp, i32, vp, i32, i32, vp]
    L.aqmb_gemv_multi.argtypes = [ctypes.POINTER(vp), i32, i32, vp, i32, i32, ctypes.POINTER(vp), i32, vp]
    L.aqmb_gemm.argtypes = [vp, i32, vp, i32, vp, i32, vp]
    L.aqmb_gemm_ws.argtypes = [vp, i32, vp, i32, vp, i32, vp, ctypes.c_size_t, vp]
    L.aqmb_gemm_workspace_bytes.argtypes = [vp, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
    L.aqmb_dequant.argtypes = [vp, i32, vp, i32, vp]
    L.aqmb_prefix_distortion.argtypes = [vp, vp, i32, vp, i32, i32, vp, vp]
    L.aqmb_prefix_distortion_noalloc.argtypes = [vp, vp, i32, vp, i32, i32, vp, vp]
    L.aqmb_beam_search.argtypes = [ctypes.POINTER(Desc), i32, i32, vp, vp, vp, vp, vp, vp]
    L.aqmb_beam_search_weighted.argtypes = [ctypes.POINTER(Desc), i32, i32, vp, vp, vp, vp, vp, vp, vp]
    i64, f32, ip = ctypes.c_int64, ctypes.c_float, ctypes.POINTER(i32)
    cp = ctypes.POINTER(KVCacheDesc)
    L.aqmb_rms_norm.argtypes = [vp, i32, i64, vp, vp, i64, vp, f32, f32, i32, i32, vp, i32, i64, vp, i32, vp]
    L.aqmb_w4_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(W4Desc), vp, vp, vp, vp]
    L.aqmb_w4_destroy.argtypes = [vp]
    L.aqmb_w4_get_desc.argtypes = [vp, ctypes.POINTER(W4Desc)]
    L.aqmb_w4_gemv.argtypes = [vp, vp, i32, i64, vp, i32, i32, vp, i32, i64, vp]
    L.aqmb_paged_attention.argtypes = [cp, vp, i32, i64, i32, vp, i64, vp, i32, i32, f32, i32, vp, i64, vp, vp,
                                       ctypes.c_size_t, vp]
    L.aqmb_paged_attention_workspace_bytes.argtypes = [cp, i32, i32, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
    L.aqmb_kv_append.argtypes = [cp, vp, i64, vp, i64, i32, vp, i32, vp]
    L.aqmb_kv_copy_pages.argtypes = [cp, i32, vp, vp, i32, vp]
    L.aqmb_pages_create.argtypes = [ctypes.POINTER(vp), i32, i32, i32]
    L.aqmb_pages_destroy.argtypes = [vp]
    L.aqmb_pages_add.argtypes = [vp, ip]
    L.aqmb_pages_fork.argtypes = [vp, i32, ip]
    L.aqmb_pages_extend.argtypes = [vp, i32, i32, vp, ip, ip]
    L.aqmb_pages_free.argtypes = [vp, i32]
    L.aqmb_pages_compact.argtypes = [vp, vp, vp, ip]
    L.aqmb_pages_table.argtypes = [vp, i32, vp, i32, ip, ip]
    L.aqmb_pages_counts.argtypes = [vp, ip, ip]
    L.aqmb_validate.argtypes = [ctypes.POINTER(Desc), i32, i32, i32, i32, i32, vp, vp]
    L.aqmb_bits_per_weight.argtypes = [ctypes.POINTER(Desc), i32]
    L.aqmb_bits_per_weight.restype = ctypes.c_double
    L.aqmb_strerror.argtypes = [i32]
    L.aqmb_strerror.restype = ctypes.c_char_p
    L.aqmb_last_error.argtypes = []
    L.aqmb_last_error.restype = ctypes.c_char_p
    for f in ("aqmb_create", "aqmb_create_prefix", "aqmb_load_planes", "aqmb_drop_planes", "aqmb_resident_planes",
              "aqmb_destroy", "aqmb_get_desc", "aqmb_gemv", "aqmb_gemv_select", "aqmb_gemv_multi", "aqmb_gemm",
              "aqmb_gemm_select", "aqmb_gemm_ws", "aqmb_gemm_workspace_bytes",
              "aqmb_dequant", "aqmb_prefix_distortion", "aqmb_prefix_distortion_noalloc", "aqmb_beam_search",
              "aqmb_beam_search_weighted",
              "aqmb_validate", "aqmb_rms_norm", "aqmb_w4_create", "aqmb_w4_destroy", "aqmb_w4_get_desc",
              "aqmb_w4_gemv", "aqmb_paged_attention", "aqmb_paged_attention_workspace_bytes", "aqmb_kv_append",
              "aqmb_kv_copy_pages", "aqmb_pages_create", "aqmb_pages_destroy", "aqmb_pages_add", "aqmb_pages_fork",
              "aqmb_pages_extend", "aqmb_pages_free", "aqmb_pages_compact", "aqmb_pages_table",
              "aqmb_pages_counts"):
        getattr(L, f).restype = st
    return L


lib = _load()

import torch  # noqa: E402  (after the library's own import of it, see _load)

# The operators between the layers take their usual calls past ctypes: _direct checks the tensors, makes the call
# and returns its status, or None where the functions below have to look. Without it they take every call.
try:
    from . import _direct  # noqa: E402
    _direct.bind(*(ctypes.cast(getattr(lib, f), ctypes.c_void_p).value for f in (
        "aqmb_rms_norm", "aqmb_w4_gemv", "aqmb_paged_attention", "aqmb_paged_attention_workspace_bytes",
        "aqmb_kv_append", "aqmb_kv_copy_pages")))
except ImportError as e:
    _direct = None
    warnings.warn(f"{os.path.join(os.path.dirname(LIB_PATH), '_direct.so')} is missing or was built for another PyTorch "
                  f"({e}): the operators between the layers go through ctypes, about 3 us a call dearer. Build it with "
                  f"python -m paper_2606_12876_amd.build", RuntimeWarning)

_TORCH_DT = {torch.float16: int(DType.F16), torch.bfloat16: int(DType.BF16), torch.float32: int(DType.F32)}
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_get_device = getattr(torch._C, "_cuda_getDevice", None)


def strerror(status: int) -> str:
    return lib.aqmb_strerror(int(status)).decode()


def last_error() -> str:
    return lib.aqmb_last_error().decode()


def _check(status: int, where: str):
    if status != Status.OK:
        raise AqmbError(status, where, last_error() or strerror(status))


def _ptr(t) -> Optional[int]:
    """Device address of a tensor (or an int address, or None)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None and _get_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_get_device())     # torch.cuda.current_stream().cuda_stream without its Stream object
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _dtype(t, default=None) -> DType:
    if isinstance(t, (DType, int)):
        return DType(t)
    return DType(_torch_dt(t))


def _torch_dt(t) -> int:
    d = _TORCH_DT.get(t.dtype)
    if d is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return d


def make_desc(d_out: int, d_in: int, num_codebooks: int, code_bits: int = 8, group_size: int = 8) -> Desc:
    return Desc(d_out, d_in, group_size, num_codebooks, code_bits)


def _nbytes(t) -> Optional[int]:
    if hasattr(t, "numel") and hasattr(t, "element_size"):
        return t.numel() * t.element_size()
    return None


def create(desc: Desc, codes, codebooks, scales, stream=None) -> int:
    """aqmb_create: codes [M][d_out][d_in/g] uint8|uint16, codebooks [M][2^B][g] fp16 bits,
    scales [d_out] fp16 bits, all device buffers. Returns the layer handle.

    The C library sees raw pointers; when tensors are passed their sizes are checked here so
    that a short buffer is rejected instead of read past its end."""
    g = desc.group_size if desc.group_size > 0 else 1
    need = {"codes": desc.num_codebooks * desc.d_out * (desc.d_in // g) * (1 if desc.code_bits <= 8 else 2),
            "codebooks": desc.num_codebooks * (1 << max(0, min(desc.code_bits, 16))) * desc.group_size * 2,
            "scales": desc.d_out * 2}
    for name, t in (("codes", codes), ("codebooks", codebooks), ("scales", scales)):
        n = _nbytes(t)
        if n is not None and n < need[name]:
            raise AqmbError(Status.EINVAL, "aqmb_create", f"{name} holds {n} bytes, the descriptor needs {need[name]}")
    h = ctypes.c_void_p()
    _check(lib.aqmb_create(ctypes.byref(h), ctypes.byref(desc), _ptr(codes), _ptr(codebooks), _ptr(scales),
                           _stream(stream)), "aqmb_create")
    return h.value


def _need_planes(desc: Desc, codes, n_planes: int, where: str):
    g = desc.group_size if desc.group_size > 0 else 1
    need = max(n_planes, 0) * desc.d_out * (desc.d_in // g) * (1 if desc.code_bits <= 8 else 2)
    n = _nbytes(codes)
    if n is not None and n < need:
        raise AqmbError(Status.EINVAL, where, f"codes holds {n} bytes, {n_planes} planes need {need}")


def create_prefix(desc: Desc, resident: int, codes, codebooks, scales, stream=None) -> int:
    """aqmb_create_prefix: a layer holding only code planes 0..resident-1 (codes [resident][d_out][d_in/g])."""
    _need_planes(desc, codes, resident, "aqmb_create_prefix")
    h = ctypes.c_void_p()
    _check(lib.aqmb_create_prefix(ctypes.byref(h), ctypes.byref(desc), resident, _ptr(codes), _ptr(codebooks),
                                  _ptr(scales), _stream(stream)), "aqmb_create_prefix")
    return h.value


def load_planes(layer: int, n_planes: int, codes, stream=None) -> None:
    """aqmb_load_planes: append the next n_planes code planes (codes [n_planes][d_out][d_in/g])."""
    _need_planes(get_desc(layer), codes, n_planes, "aqmb_load_planes")
    _check(lib.aqmb_load_planes(layer, n_planes, _ptr(codes), _stream(stream)), "aqmb_load_planes")


def drop_planes(layer: int, keep: int) -> None:
    """aqmb_drop_planes: keep code planes 0..keep-1 and free the others."""
    _check(lib.aqmb_drop_planes(layer, keep), "aqmb_drop_planes")


def resident_planes(layer: int) -> int:
    r = ctypes.c_int32()
    _check(lib.aqmb_resident_planes(layer, ctypes.byref(r)), "aqmb_resident_planes")
    return r.value


def destroy(layer: int) -> None:
    _check(lib.aqmb_destroy(layer), "aqmb_destroy")


def get_desc(layer: int) -> Desc:
    d = Desc()
    _check(lib.aqmb_get_desc(layer, ctypes.byref(d)), "aqmb_get_desc")
    return d


_ELEM = {0: 2, 1: 2, 2: 4}


def _need(t, n_elems: int, dtype, what: str, where: str):
    n = _nbytes(t)
    if n is not None and int(dtype) in _ELEM and n < n_elems * _ELEM[int(dtype)]:
        raise AqmbError(Status.EINVAL, where, f"{what} holds {n} bytes, needs {n_elems * _ELEM[int(dtype)]}")


def gemv(layer: int, k: int, x, x_dtype, batch: int, y, y_dtype, stream=None) -> None:
    d = get_desc(layer)
    if 1 <= batch <= 16:
        _need(x, batch * d.d_in, x_dtype, "x", "aqmb_gemv")
        _need(y, batch * d.d_out, y_dtype, "y", "aqmb_gemv")
    _check(lib.aqmb_gemv(layer, k, _ptr(x), int(x_dtype), batch, _ptr(y), int(y_dtype), _stream(stream)),
           "aqmb_gemv")


def gemv_select(layer: int, k: int, x, x_dtype, batch: int, y, y_dtype, kernel, stream=None) -> None:
    """aqmb_gemv_select: aqmb_gemv with the kernel named by ``kernel`` (a GemvKernel)."""
    d = get_desc(layer)
    if 1 <= batch <= 16:
        _need(x, batch * d.d_in, x_dtype, "x", "aqmb_gemv_select")
        _need(y, batch * d.d_out, y_dtype, "y", "aqmb_gemv_select")
    _check(lib.aqmb_gemv_select(layer, k, _ptr(x), int(x_dtype), batch, _ptr(y), int(y_dtype), int(kernel),
                                _stream(stream)), "aqmb_gemv_select")


MAX_MULTI = 16


def gemv_multi(layers, k: int, x, x_dtype, batch: int, ys, y_dtype, stream=None) -> None:
    """aqmb_gemv_multi: the GEMV of every layer in `layers` (same d_in) on the same x, one output each."""
    layers, ys = list(layers), list(ys)
    if len(layers) != len(ys):
        raise AqmbError(Status.EINVAL, "aqmb_gemv_multi", "one output per layer")
    if 1 <= batch <= 16 and 1 <= len(layers) <= MAX_MULTI:
        for layer, y in zip(layers, ys):
            d = get_desc(layer)
            _need(x, batch * d.d_in, x_dtype, "x", "aqmb_gemv_multi")
            _need(y, batch * d.d_out, y_dtype, "y", "aqmb_gemv_multi")
    n = len(layers)
    la = (ctypes.c_void_p * max(n, 1))(*[ctypes.c_void_p(h) for h in layers])
    ya = (ctypes.c_void_p * max(n, 1))(*[ctypes.c_void_p(_ptr(y)) for y in ys])
    _check(lib.aqmb_gemv_multi(la, n, k, _ptr(x), int(x_dtype), batch, ya, int(y_dtype), _stream(stream)),
           "aqmb_gemv_multi")


def gemm(layer: int, k: int, X, n_tokens: int, Y, y_dtype, stream=None) -> None:
    d = get_desc(layer)
    if n_tokens >= 1:
        _need(X, n_tokens * d.d_in, DType.BF16, "X", "aqmb_gemm")
        _need(Y, n_tokens * d.d_out, y_dtype, "Y", "aqmb_gemm")
    _check(lib.aqmb_gemm(layer, k, _ptr(X), n_tokens, _ptr(Y), int(y_dtype), _stream(stream)), "aqmb_gemm")


def gemm_select(layer: int, k: int, X, n_tokens: int, Y, y_dtype, tiling, stream=None) -> None:
    """aqmb_gemm_select: aqmb_gemm with the tiling named by ``tiling`` (a GemmTiling)."""
    d = get_desc(layer)
    if n_tokens >= 1:
        _need(X, n_tokens * d.d_in, DType.BF16, "X", "aqmb_gemm_select")
        _need(Y, n_tokens * d.d_out, y_dtype, "Y", "aqmb_gemm_select")
    _check(lib.aqmb_gemm_select(layer, k, _ptr(X), n_tokens, _ptr(Y), int(y_dtype), int(tiling), _stream(stream)),
           "aqmb_gemm_select")


def gemm_workspace_bytes(layer: int, k: int, n_tokens: int) -> int:
    """aqmb_gemm_workspace_bytes: the workspace gemm_ws needs for its two-pass path (0: not taken)."""
    n = ctypes.c_size_t(0)
    _check(lib.aqmb_gemm_workspace_bytes(layer, k, n_tokens, ctypes.byref(n)), "aqmb_gemm_workspace_bytes")
    return n.value


def gemm_ws(layer: int, k: int, X, n_tokens: int, Y, y_dtype, workspace, stream=None) -> None:
    """aqmb_gemm_ws: aqmb_gemm with a caller-owned device workspace (a tensor, or None)."""
    d = get_desc(layer)
    if n_tokens >= 1:
        _need(X, n_tokens * d.d_in, DType.BF16, "X", "aqmb_gemm_ws")
        _need(Y, n_tokens * d.d_out, y_dtype, "Y", "aqmb_gemm_ws")
    nb = _nbytes(workspace) if workspace is not None else 0
    _check(lib.aqmb_gemm_ws(layer, k, _ptr(X), n_tokens, _ptr(Y), int(y_dtype), _ptr(workspace), nb or 0,
                            _stream(stream)), "aqmb_gemm_ws")


def dequant(layer: int, k: int, W, w_dtype, stream=None) -> None:
    d = get_desc(layer)
    _need(W, d.d_out * d.d_in, w_dtype, "W", "aqmb_dequant")
    _check(lib.aqmb_dequant(layer, k, _ptr(W), int(w_dtype), _stream(stream)), "aqmb_dequant")


def prefix_distortion(layer: int, W, w_dtype, Xt, x_dtype, n: int, D, stream=None) -> None:
    """aqmb_prefix_distortion: D[k-1] = ||(W - W_k) X||_F^2 / (d_out n) for k = 1..M, with the n
    calibration inputs as the rows of Xt [n][d_in] (fp16) and W [d_out][d_in] fp16; D holds M
    float64 values in device memory."""
    d = get_desc(layer)
    _need(W, d.d_out * d.d_in, w_dtype, "W", "aqmb_prefix_distortion")
    if n >= 1:
        _need(Xt, n * d.d_in, x_dtype, "Xt", "aqmb_prefix_distortion")
    nd = _nbytes(D)
    need = 8 * resident_planes(layer)
    if nd is not None and nd < need:
        raise AqmbError(Status.EINVAL, "aqmb_prefix_distortion", f"D holds {nd} bytes, needs {need}")
    _check(lib.aqmb_prefix_distortion(layer, _ptr(W), int(w_dtype), _ptr(Xt), int(x_dtype), n, _ptr(D),
                                      _stream(stream)), "aqmb_prefix_distortion")


def prefix_distortion_noalloc(layer: int, W, w_dtype, Xt, x_dtype, n: int, D, stream=None) -> None:
    """aqmb_prefix_distortion_noalloc: prefix_distortion with the library's fixed scratch (no device
    allocation; calls that overlap on one device race)."""
    d = get_desc(layer)
    _need(W, d.d_out * d.d_in, w_dtype, "W", "aqmb_prefix_distortion_noalloc")
    if n >= 1:
        _need(Xt, n * d.d_in, x_dtype, "Xt", "aqmb_prefix_distortion_noalloc")
    nd = _nbytes(D)
    need = 8 * resident_planes(layer)
    if nd is not None and nd < need:
        raise AqmbError(Status.EINVAL, "aqmb_prefix_distortion_noalloc", f"D holds {nd} bytes, needs {need}")
    _check(lib.aqmb_prefix_distortion_noalloc(layer, _ptr(W), int(w_dtype), _ptr(Xt), int(x_dtype), n, _ptr(D),
                                              _stream(stream)), "aqmb_prefix_distortion_noalloc")


MAX_BEAM = 16


def beam_search(desc: Desc, k: int, beam: int, W, codebooks, scales, codes, errors=None, stream=None) -> None:
    """aqmb_beam_search: codes [k][d_out][d_in/8] uint8 (and errors [d_out][d_in/8] float32 if given)
    from a beam search over codebooks 0..k-1 for every group of W [d_out][d_in] fp16."""
    G = desc.d_in // max(desc.group_size, 1)
    _need(W, desc.d_out * desc.d_in, DType.F16, "W", "aqmb_beam_search")
    nc = _nbytes(codes)
    if nc is not None and 1 <= k and nc < k * desc.d_out * G:
        raise AqmbError(Status.EINVAL, "aqmb_beam_search", f"codes holds {nc} bytes, needs {k * desc.d_out * G}")
    ne = _nbytes(errors) if errors is not None else None
    if ne is not None and ne < 4 * desc.d_out * G:
        raise AqmbError(Status.EINVAL, "aqmb_beam_search", f"errors holds {ne} bytes, needs {4 * desc.d_out * G}")
    _check(lib.aqmb_beam_search(ctypes.byref(desc), k, beam, _ptr(W), _ptr(codebooks), _ptr(scales), _ptr(codes),
                                _ptr(errors) if errors is not None else None, _stream(stream)), "aqmb_beam_search")


def beam_search_weighted(desc: Desc, k: int, beam: int, W, codebooks, scales, H, codes, errors=None,
                         stream=None) -> None:
    """aqmb_beam_search_weighted: the code search with the data-aware error d^T H_j d; H is
    [d_in/8][8][8] float32 (the symmetric diagonal blocks of X X^T / n)."""
    G = desc.d_in // max(desc.group_size, 1)
    _need(W, desc.d_out * desc.d_in, DType.F16, "W", "aqmb_beam_search_weighted")
    _need(H, G * 64, DType.F32, "H", "aqmb_beam_search_weighted")
    nc = _nbytes(codes)
    if nc is not None and 1 <= k and nc < k * desc.d_out * G:
        raise AqmbError(Status.EINVAL, "aqmb_beam_search_weighted", f"codes holds {nc} bytes, needs {k * desc.d_out * G}")
    ne = _nbytes(errors) if errors is not None else None
    if ne is not None and ne < 4 * desc.d_out * G:
        raise AqmbError(Status.EINVAL, "aqmb_beam_search_weighted", f"errors holds {ne} bytes, needs {4 * desc.d_out * G}")
    _check(lib.aqmb_beam_search_weighted(ctypes.byref(desc), k, beam, _ptr(W), _ptr(codebooks), _ptr(scales), _ptr(H),
                                         _ptr(codes), _ptr(errors) if errors is not None else None, _stream(stream)),
           "aqmb_beam_search_weighted")


def bits_per_weight(desc: Desc, k: int) -> float:
    return float(lib.aqmb_bits_per_weight(ctypes.byref(desc), k))


def validate(desc: Desc, op: int, k: int, n: int, in_dtype, out_dtype, inp, out) -> Status:
    return Status(lib.aqmb_validate(ctypes.byref(desc), op, k, n, int(in_dtype), int(out_dtype), _ptr(inp), _ptr(out)))


class QuantLinear:
    """A quantized linear layer y = x . W_k^T served at any precision level k <= M.

    Holds the library's layer handle. ``forward`` allocates the output with PyTorch and calls the
    library on the current stream: up to 16 input rows go to aqmb_gemv (fp16 or bf16 x), more
    rows to aqmb_gemm, which takes bf16 x only (other dtypes are refused, not converted: the
    binding only marshals arguments). The code width B follows from the codebooks: 16, 256 or
    65536 codewords give 4-, 8- or 16-bit codes (4-bit codes are passed one per byte, 0..15).
    """

    _BITS = {16: 4, 256: 8, 65536: 16}

    def __init__(self, codes, codebooks, scales, group_size: int = 8):
        M, d_out, n_groups = codes.shape
        n_cw = int(codebooks.shape[1])
        if n_cw not in self._BITS:
            raise AqmbError(Status.EUNSUPPORTED, "QuantLinear", f"codebooks of {n_cw} codewords (16, 256 or 65536)")
        code_bits = self._BITS[n_cw]
        want = torch.int16 if code_bits == 16 else torch.uint8
        if codes.dtype not in ((torch.int16, torch.uint16) if code_bits == 16 else (torch.uint8,)):
            raise AqmbError(Status.EINVAL, "QuantLinear", f"codes of dtype {codes.dtype} for {code_bits}-bit codes")
        self.desc = make_desc(d_out, n_groups * group_size, M, code_bits, group_size)
        self.handle = create(self.desc, codes.contiguous().view(want), codebooks.contiguous().view(torch.int16),
                             scales.contiguous().view(torch.int16))
        self.M, self.d_out, self.d_in, self.code_bits = M, d_out, n_groups * group_size, code_bits

    def forward(self, x, k: int, out_dtype=None):
        # The library is called directly: the sizes that gemv and gemm check hold here by construction.
        d_in, d_out = self.d_in, self.d_out
        flat = x.dim() == 2 and x.shape[1] == d_in and x.is_contiguous()
        x2 = x if flat else x.reshape(-1, d_in).contiguous()
        n = x2.shape[0]
        if n > 16 and x2.dtype != torch.bfloat16:
            raise AqmbError(Status.EUNSUPPORTED, "QuantLinear",
                            f"{n} rows go to aqmb_gemm, which takes bf16 x only (got {x2.dtype})")
        y = torch.empty((n, d_out), dtype=out_dtype or x.dtype, device=x.device)
        if n <= 16:
            st = lib.aqmb_gemv(self.handle, k, x2.data_ptr(), _torch_dt(x2), n, y.data_ptr(), _torch_dt(y), _stream(None))
            if st:
                _check(st, "aqmb_gemv")
        else:
            ws = self._workspace(k, n, x.device)
            st = lib.aqmb_gemm_ws(self.handle, k, x2.data_ptr(), n, y.data_ptr(), _torch_dt(y),
                                  None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(), _stream(None))
            if st:
                _check(st, "aqmb_gemm")
        return y if flat else y.reshape(*x.shape[:-1], d_out)

    def _workspace(self, k: int, n: int, device):
        """The two-pass GEMM's workspace for this call (from PyTorch's allocator, given back to it
        when the call returns: launches on this stream keep its order), or None where aqmb_gemm is
        to run: the path does not apply, or there is no memory for it. Both give the same result
        (2048 x 4096 x 4096, k = 4: 94 us in one pass, 80 us in two)."""
        nb = ctypes.c_size_t(0)
        if n <= 144 or lib.aqmb_gemm_workspace_bytes(self.handle, k, n, ctypes.byref(nb)) != 0 or nb.value == 0:
            return None
        try:
            return torch.empty((nb.value,), dtype=torch.uint8, device=device)
        except torch.OutOfMemoryError:
            return None

    __call__ = forward

    def dequant(self, k: int, dtype=None):
        W = torch.empty((self.d_out, self.d_in), dtype=dtype or torch.float16, device="cuda")
        dequant(self.handle, k, W, _dtype(W))
        return W

    def close(self):
        if self.handle:
            destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ------------------------------------------------------------------------------------------------
# The operators between the layers. These take tensors: types, sizes and strides come from them, and
# what the library cannot see (a tensor's size and device) is checked here.
_TORCH_DT8 = {**_TORCH_DT, torch.float8_e4m3fn: int(DType.F8), torch.int8: int(DType.I8)}


def _refuse(where: str, message: str, status: Status = Status.EINVAL):
    raise AqmbError(status, where, message)


def _dt8(t, what: str, where: str) -> int:
    d = _TORCH_DT8.get(t.dtype)
    if d is None:
        _refuse(where, f"{what} has dtype {t.dtype}", Status.EUNSUPPORTED)
    return d


_current_device = _get_device if _get_device is not None else torch.cuda.current_device


def _here(where: str, **tensors) -> None:
    """Every tensor lives on the current device."""
    dev = _current_device()
    for what, t in tensors.items():
        if t is not None and t.get_device() != dev:
            _refuse(where, f"{what} is on {t.device}, device {dev} is current")


def _rows(t, rows: int, cols: int, what: str, where: str) -> int:
    """The row stride of a [rows][cols] tensor whose rows are dense (of one row: the row itself)."""
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        _refuse(where, f"{what} is {tuple(t.shape)}, not ({rows}, {cols})")
    s0, s1 = t.stride()
    if s1 != 1 and cols != 1:
        _refuse(where, f"{what}: the elements of a row must be adjacent")
    return cols if rows == 1 else s0


def _dense(t, dtype, n: int, what: str, where: str) -> None:
    if t.dtype != dtype or t.numel() != n or not t.is_contiguous():
        _refuse(where, f"{what} must be dense, of {n} elements of {dtype}")


def rms_norm(x, weight, y, *, eps: float, weight_offset: float = 0.0, residual=None, residual_out=None, scales=None,
             scale_group: int = 0, stream=None) -> None:
    """aqmb_rms_norm: y = rms_norm(x + residual) * (weight + weight_offset) for the rows of x
    [rows][cols] fp16 or bf16; y is a tensor of the same shape: fp16, bf16, fp32, or (with scales
    [rows][ceil(cols / scale_group)] fp32; scale_group 0 is the whole row) float8_e4m3fn or int8.
    With a residual, x + residual is rounded into residual_out."""
    where = "aqmb_rms_norm"
    if stream is None and _direct is not None:
        st = _direct.rms_norm(x, weight, y, eps, weight_offset, residual, residual_out, scales, scale_group)
        if st is not None:
            return _check(st, where) if st else None
    shape, dtype, dev = x.shape, x.dtype, _current_device()
    if len(shape) != 2:
        _refuse(where, f"x is {tuple(shape)}, not (rows, cols)")
    rows, cols = shape
    dt, ydt = _TORCH_DT8.get(dtype), _TORCH_DT8.get(y.dtype)
    if dt is None or ydt is None:
        _refuse(where, f"x of {dtype}, y of {y.dtype}", Status.EUNSUPPORTED)
    if x.get_device() != dev or weight.get_device() != dev or y.get_device() != dev:
        _here(where, x=x, weight=weight, y=y)
    xs = cols if x.is_contiguous() else _rows(x, rows, cols, "x", where)
    ys = cols if y.shape == shape and y.is_contiguous() else _rows(y, rows, cols, "y", where)
    if weight.dtype != dtype or weight.numel() != cols or not weight.is_contiguous():
        _dense(weight, dtype, cols, "weight", where)
    rs, rp, ro, sp = 0, None, None, None
    if residual is not None:
        if residual_out is None or residual.dtype != dtype or residual_out.dtype != dtype:
            _refuse(where, "residual and residual_out go together, in the type of x")
        if residual.get_device() != dev or residual_out.get_device() != dev:
            _here(where, residual=residual, residual_out=residual_out)
        if residual.shape == shape == residual_out.shape and residual.is_contiguous() and residual_out.is_contiguous():
            rs = cols
        else:
            rs = _rows(residual, rows, cols, "residual", where)
            if _rows(residual_out, rows, cols, "residual_out", where) != rs:
                _refuse(where, "residual and residual_out have different row strides")
        rp, ro = residual.data_ptr(), residual_out.data_ptr()
    elif residual_out is not None:
        _refuse(where, "residual and residual_out go together, in the type of x")
    if scales is not None:
        if scale_group < 0:
            _refuse(where, f"scale_group = {scale_group}")
        if scales.get_device() != dev:
            _here(where, scales=scales)
        _dense(scales, torch.float32, rows * (-(-cols // scale_group) if scale_group else 1), "scales", where)
        sp = scales.data_ptr()
    st = lib.aqmb_rms_norm(x.data_ptr(), dt, xs, rp, ro, rs, weight.data_ptr(), weight_offset, eps, rows, cols,
                           y.data_ptr(), ydt, ys, sp, scale_group,
                           _raw_stream(dev) if stream is None and _raw_stream is not None else _stream(stream))
    if st:
        _check(st, where)


def w4_create(d_out: int, d_in: int, group_size: int, weights, scales, zeros=None, stream=None) -> int:
    """aqmb_w4_create: weights [d_out][ceil(d_in/2)] uint8 (low nibble first), scales
    [d_out][ceil(d_in/group_size)] fp16, zeros the same shape uint8 or None (8). Returns the handle."""
    where = "aqmb_w4_create"
    if d_out < 1 or d_in < 1 or group_size < 1:
        _refuse(where, f"d_out = {d_out}, d_in = {d_in} and group_size = {group_size} must be >= 1")
    groups = -(-d_in // group_size)
    _here(where, weights=weights, scales=scales, zeros=zeros)
    _dense(weights, torch.uint8, d_out * ((d_in + 1) // 2), "weights", where)
    _dense(scales, torch.float16, d_out * groups, "scales", where)
    if zeros is not None:
        _dense(zeros, torch.uint8, d_out * groups, "zeros", where)
    h = ctypes.c_void_p()
    desc = W4Desc(d_out, d_in, group_size)
    _check(lib.aqmb_w4_create(ctypes.byref(h), ctypes.byref(desc), _ptr(weights), _ptr(scales), _ptr(zeros),
                              _stream(stream)), where)
    return h.value


def w4_destroy(layer: int) -> None:
    _check(lib.aqmb_w4_destroy(layer), "aqmb_w4_destroy")


def w4_get_desc(layer: int) -> W4Desc:
    d = W4Desc()
    _check(lib.aqmb_w4_get_desc(layer, ctypes.byref(d)), "aqmb_w4_get_desc")
    return d


def _w4_gemv(layer: int, d_out: int, d_in: int, group_size: int, x, y, x_scales, stream) -> None:
    where = "aqmb_w4_gemv"
    if stream is None and _direct is not None:
        st = _direct.w4_gemv(layer, d_out, d_in, group_size, x, y, x_scales)
        if st is not None:
            return _check(st, where) if st else None
    shape, yshape = x.shape, y.shape
    if len(shape) != 2:
        _refuse(where, f"x is {tuple(shape)}, not (batch, d_in)")
    batch, cols = shape
    dt, ydt = _TORCH_DT8.get(x.dtype), _TORCH_DT8.get(y.dtype)
    if dt is None or ydt is None:
        _refuse(where, f"x of {x.dtype}, y of {y.dtype}", Status.EUNSUPPORTED)
    dev, group, sp = _current_device(), 0, None
    if x.get_device() != dev or y.get_device() != dev:
        _here(where, x=x, y=y)
    xs = cols if cols == d_in and x.is_contiguous() else _rows(x, batch, d_in, "x", where)
    ys = d_out if yshape == (batch, d_out) and y.is_contiguous() else _rows(y, batch, d_out, "y", where)
    if x_scales is not None:
        # One scale per row, or one per group (the same thing where a row is one group).
        if x_scales.numel() != batch:
            group = group_size
        if x_scales.get_device() != dev:
            _here(where, x_scales=x_scales)
        _dense(x_scales, torch.float32, batch * (-(-d_in // group_size) if group else 1), "x_scales", where)
        sp = x_scales.data_ptr()
    st = lib.aqmb_w4_gemv(layer, x.data_ptr(), dt, xs, sp, group, batch, y.data_ptr(), ydt, ys,
                          _raw_stream(dev) if stream is None and _raw_stream is not None else _stream(stream))
    if st:
        _check(st, where)


def w4_gemv(layer: int, x, y, x_scales=None, stream=None) -> None:
    """aqmb_w4_gemv: y [batch][d_out] = x [batch][d_in] times the layer's weights, 1 <= batch <= 16; x
    fp16, bf16, or float8_e4m3fn / int8 with x_scales [batch][1] or [batch][groups of the layer] fp32."""
    d = w4_get_desc(layer)
    _w4_gemv(layer, d.d_out, d.d_in, d.group_size, x, y, x_scales, stream)


class W4Linear:
    """A linear layer of 4-bit weights with group scales, y = x W^T for up to 16 rows of x.

    weights [d_out][ceil(d_in/2)] uint8, scales [d_out][groups] fp16, zeros [d_out][groups] uint8 or
    None; d_in defaults to 2 * weights.shape[1]. ``gemv`` writes into a given y, ``forward`` (and a
    call) allocates it, in the type of x or out_dtype (8-bit x: bf16)."""

    def __init__(self, weights, scales, zeros=None, *, d_in: Optional[int] = None, group_size: int = 128):
        self.handle = None
        if weights.dim() != 2:
            _refuse("W4Linear", f"weights are {tuple(weights.shape)}, not (d_out, ceil(d_in / 2))")
        self.d_out, self.d_in = weights.shape[0], 2 * weights.shape[1] if d_in is None else d_in
        self.group_size = group_size
        self.handle = w4_create(self.d_out, self.d_in, group_size, weights, scales, zeros)

    def gemv(self, x, y, x_scales=None, stream=None) -> None:
        _w4_gemv(self.handle, self.d_out, self.d_in, self.group_size, x, y, x_scales, stream)

    def forward(self, x, x_scales=None, out_dtype=None):
        x2 = x if x.dim() == 2 and x.stride(-1) == 1 else x.reshape(-1, x.shape[-1]).contiguous()
        dt = out_dtype or (x.dtype if x.dtype in _TORCH_DT else torch.bfloat16)
        y = torch.empty((x2.shape[0], self.d_out), dtype=dt, device=x.device)
        self.gemv(x2, y, x_scales)
        return y if x.dim() == 2 else y.reshape(*x.shape[:-1], self.d_out)

    __call__ = forward

    def close(self):
        if self.handle:
            w4_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class KVCache:
    """A paged key-value cache of one attention layer over tensors of the caller.

    k, v: [n_pages][n_kv_heads][page_size][head_dim] (layout "head") or
    [n_pages][page_size][n_kv_heads][head_dim] ("slot"), dense inside a page: fp16, bf16, or
    float8_e4m3fn with k_scale, v_scale fp32 of the same shape without head_dim, dense. ``allocate``
    makes the tensors. The methods take the arguments of paged_attention and kv_append."""

    _LAYOUTS = {"head": KVLayout.HEAD_MAJOR, "slot": KVLayout.SLOT_MAJOR}

    def __init__(self, k, v, k_scale=None, v_scale=None, *, layout: str = "head"):
        where = "KVCache"
        if layout not in self._LAYOUTS:
            _refuse(where, f"layout {layout!r} is not 'head' or 'slot'")
        dt = _TORCH_DT8.get(k.dtype)
        if dt not in (DType.F16, DType.BF16, DType.F8):
            _refuse(where, f"k has dtype {k.dtype}", Status.EUNSUPPORTED)
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.stride() != v.stride():
            _refuse(where, "k and v must be 4-dimensional, alike in shape, type and strides")
        if 0 in k.shape:
            _refuse(where, f"an empty cache {tuple(k.shape)}")
        page = k[0].numel()
        if not k[0].is_contiguous() or (k.shape[0] > 1 and k.stride(0) < page):
            _refuse(where, "a page must be dense")
        n = k.shape[0] * k.shape[1] * k.shape[2]
        if (dt == DType.F8) != (k_scale is not None) or (k_scale is None) != (v_scale is None):
            _refuse(where, "an 8-bit cache, and no other, has k_scale and v_scale")
        for what, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            if t is not None:
                _dense(t, torch.float32, n, what, where)
                if t.device != k.device:
                    _refuse(where, f"{what} is on {t.device}, k on {k.device}")
        if not k.is_cuda or v.device != k.device:
            _refuse(where, "k and v must be on one GPU")
        lay = self._LAYOUTS[layout]
        heads, size = (k.shape[1], k.shape[2]) if lay == KVLayout.HEAD_MAJOR else (k.shape[2], k.shape[1])
        self.k, self.v, self.k_scale, self.v_scale, self.layout = k, v, k_scale, v_scale, layout
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k.shape[0], heads, size, k.shape[3]
        self.device_index = k.get_device()
        self.desc = KVCacheDesc(k.data_ptr(), v.data_ptr(), _ptr(k_scale), _ptr(v_scale),
                                k.stride(0) if k.shape[0] > 1 else page, int(dt), int(lay), k.shape[0], size, heads,
                                k.shape[3])
        self._ref = ctypes.byref(self.desc)
        self._address = ctypes.addressof(self.desc)
        self._plans = {}

    @classmethod
    def allocate(cls, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, dtype=torch.bfloat16, *,
                 layout: str = "head", device="cuda") -> "KVCache":
        a, b = (n_kv_heads, page_size) if layout == "head" else (page_size, n_kv_heads)
        k, v = (torch.empty((n_pages, a, b, head_dim), dtype=dtype, device=device) for _ in range(2))
        ks, vs = (torch.empty((n_pages, a, b), dtype=torch.float32, device=device) if dtype == torch.float8_e4m3fn
                  else None for _ in range(2))
        return cls(k, v, ks, vs, layout=layout)

    def _current(self, where: str) -> None:
        dev = _current_device()
        if dev != self.device_index:
            _refuse(where, f"the cache is on device {self.device_index}, device {dev} is current")

    def workspace_bytes(self, n_heads: int, n_seqs: int, max_length: int, window: int = 0) -> int:
        """aqmb_paged_attention_workspace_bytes (a function of these numbers, so asked once for each)."""
        key = (n_heads, n_seqs, max_length, window)
        n = self._plans.get(key)
        if n is None:
            b = ctypes.c_size_t(0)
            _check(lib.aqmb_paged_attention_workspace_bytes(self._ref, n_heads, n_seqs, max_length, window,
                                                            ctypes.byref(b)), "aqmb_paged_attention_workspace_bytes")
            if len(self._plans) >= 4096:
                self._plans.clear()
            n = self._plans[key] = b.value
        return n

    def attention(self, q, page_table, lengths, out, *, scale: float, max_length: Optional[int] = None,
                  window: int = 0, lse=None, workspace=None, stream=None) -> None:
        """aqmb_paged_attention: out [n_seqs][n_heads][head_dim] for one query token of every sequence;
        page_table [n_seqs][pages] and lengths [n_seqs] int32 on the GPU. max_length bounds the lengths
        (default: what the table holds). Without a workspace one is taken from PyTorch's allocator on the
        call's stream."""
        where = "aqmb_paged_attention"
        if stream is None and _direct is not None:
            st = _direct.paged_attention(self._address, self.device_index, q, page_table, lengths, out, scale, max_length,
                                         window, lse, workspace)
            if st is not None:
                return _check(st, where) if st else None
        dev = _current_device()
        if dev != self.device_index:
            self._current(where)
        if q.get_device() != dev or page_table.get_device() != dev or lengths.get_device() != dev \
                or out.get_device() != dev:
            _here(where, q=q, page_table=page_table, lengths=lengths, out=out)
        shape, dtype, tshape = q.shape, q.dtype, page_table.shape
        if len(shape) != 3 or shape[2] != self.head_dim:
            _refuse(where, f"q is {tuple(shape)}, not (n_seqs, n_heads, {self.head_dim})")
        n, heads, dim = shape
        row = heads * dim
        if out.shape != shape or out.dtype != dtype:
            _refuse(where, f"out is {tuple(out.shape)} of {out.dtype}, not {tuple(shape)} of {dtype}")
        qs = row if q.is_contiguous() else self._stride(q, n, row, "q", where)
        os_ = row if out.is_contiguous() else self._stride(out, n, row, "out", where)
        if len(tshape) != 2 or tshape[0] != n or page_table.dtype != torch.int32 \
                or (not page_table.is_contiguous() and tshape[1] > 1 and page_table.stride(1) != 1):
            _refuse(where, f"page_table must be int32 [{n}][pages] with dense rows")
        if lengths.dtype != torch.int32 or lengths.numel() != n or not lengths.is_contiguous():
            _dense(lengths, torch.int32, n, "lengths", where)
        lp = None
        if lse is not None:
            if lse.get_device() != dev:
                _here(where, lse=lse)
            _dense(lse, torch.float32, n * heads, "lse", where)
            lp = lse.data_ptr()
        per = tshape[1]
        if max_length is None:
            max_length = min(per * self.page_size, 1 << 27)
        elif max_length > per * self.page_size:
            _refuse(where, f"max_length = {max_length} needs more pages than the table's {per}")
        need = self.workspace_bytes(heads, n, max_length, window)
        wp, wb = None, 0
        if workspace is not None:
            _here(where, workspace=workspace)
            if not workspace.is_contiguous():
                _refuse(where, "workspace must be dense")
            wp, wb = workspace.data_ptr(), _nbytes(workspace)
        elif need:
            if stream is None:
                workspace = torch.empty((need,), dtype=torch.uint8, device=q.device)
            else:   # the allocator ties memory to the stream that is current
                s = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream)
                with torch.cuda.stream(s):
                    workspace = torch.empty((need,), dtype=torch.uint8, device=q.device)
            wp, wb = workspace.data_ptr(), need
        st = lib.aqmb_paged_attention(self._ref, q.data_ptr(), _dt8(q, "q", where), qs, heads, page_table.data_ptr(),
                                      page_table.stride(0) if n > 1 else per, lengths.data_ptr(), n, max_length, scale,
                                      window, out.data_ptr(), os_, lp, wp, wb,
                                      _raw_stream(dev) if stream is None and _raw_stream is not None else _stream(stream))
        if st:
            _check(st, where)

    @staticmethod
    def _stride(t, n: int, row: int, what: str, where: str) -> int:
        """The stride between the rows [heads][head_dim] of a 3-dimensional tensor, which must be dense."""
        if t.numel() and ((t.stride(2) != 1 and t.shape[2] != 1) or (t.stride(1) != t.shape[2] and t.shape[1] != 1)):
            _refuse(where, f"{what}: the heads of a row must be dense")
        return t.stride(0) if n > 1 else row

    def append(self, k, v, slots, stream=None) -> None:
        """aqmb_kv_append: write k, v [n_tokens][n_kv_heads][head_dim] (fp16 or bf16) into slots int64
        [n_tokens] on the GPU (page * page_size + offset; outside the cache: skipped)."""
        where = "aqmb_kv_append"
        if stream is None and _direct is not None:
            st = _direct.kv_append(self._address, self.device_index, k, v, slots)
            if st is not None:
                return _check(st, where) if st else None
        dev = _current_device()
        if dev != self.device_index:
            self._current(where)
        if k.get_device() != dev or v.get_device() != dev or slots.get_device() != dev:
            _here(where, k=k, v=v, slots=slots)
        n, dim, heads = slots.numel(), self.head_dim, self.n_kv_heads
        if slots.dtype != torch.int64 or not slots.is_contiguous():
            _dense(slots, torch.int64, n, "slots", where)
        shape, dtype, row = k.shape, k.dtype, heads * dim
        if shape != (n, heads, dim) or v.shape != shape or v.dtype != dtype:
            _refuse(where, f"k is {tuple(shape)} of {dtype} and v {tuple(v.shape)} of {v.dtype}, not ({n}, {heads}, {dim})")
        ks = row if k.is_contiguous() else self._stride(k, n, row, "k", where)
        vs = row if v.is_contiguous() else self._stride(v, n, row, "v", where)
        st = lib.aqmb_kv_append(self._ref, k.data_ptr(), ks, v.data_ptr(), vs, _dt8(k, "k", where), slots.data_ptr(), n,
                                _raw_stream(dev) if stream is None and _raw_stream is not None else _stream(stream))
        if st:
            _check(st, where)


def paged_attention(cache: KVCache, q, page_table, lengths, out, **kw) -> None:
    """aqmb_paged_attention (see KVCache.attention)."""
    cache.attention(q, page_table, lengths, out, **kw)


def paged_attention_workspace_bytes(cache: KVCache, n_heads: int, n_seqs: int, max_length: int, window: int = 0) -> int:
    return cache.workspace_bytes(n_heads, n_seqs, max_length, window)


def kv_append(cache: KVCache, k, v, slots, stream=None) -> None:
    """aqmb_kv_append (see KVCache.append)."""
    cache.append(k, v, slots, stream)


def kv_copy_pages(caches, src, dst, stream=None) -> None:
    """aqmb_kv_copy_pages: page src[i] to page dst[i] (int32, on the GPU) in every KVCache of `caches`."""
    where = "aqmb_kv_copy_pages"
    if not isinstance(caches, (list, tuple)):
        caches = list(caches)
    if stream is None and _direct is not None:
        st = _direct.kv_copy_pages(caches, src, dst)
        if st is not None:
            return _check(st, where) if st else None
    _here(where, src=src, dst=dst)
    for c in caches:
        c._current(where)
    n = src.numel()
    _dense(src, torch.int32, n, "src", where)
    _dense(dst, torch.int32, n, "dst", where)
    descs = (KVCacheDesc * max(len(caches), 1))(*[c.desc for c in caches])
    st = lib.aqmb_kv_copy_pages(descs, len(caches), src.data_ptr(), dst.data_ptr(), n, _stream(stream))
    if st:
        _check(st, where)


class PagePool:
    """aqmb_pages_*: which pages of a cache each sequence holds, on the host. Sequences are small integers.

    extend returns (slots int64 tensor, copies) where copies is [] or [(src, dst)]: the page to copy in
    every layer's cache before the tokens are written, and before the next fork, free or compact (the pairs of
    extends in a row may be copied together); compact returns such a list for the whole pool.
    table returns the pages as an int32 tensor. All of them are CPU tensors and lists: one upload of a
    step's tables, slots and copies serves all layers."""

    def __init__(self, n_pages: int, page_size: int, max_seqs: int):
        self.handle = None
        h = ctypes.c_void_p()
        _check(lib.aqmb_pages_create(ctypes.byref(h), n_pages, page_size, max_seqs), "aqmb_pages_create")
        self.handle, self.n_pages, self.page_size, self.max_seqs = h.value, n_pages, page_size, max_seqs

    def add(self) -> int:
        s = ctypes.c_int()
        _check(lib.aqmb_pages_add(self.handle, ctypes.byref(s)), "aqmb_pages_add")
        return s.value

    def fork(self, seq: int) -> int:
        s = ctypes.c_int()
        _check(lib.aqmb_pages_fork(self.handle, seq, ctypes.byref(s)), "aqmb_pages_fork")
        return s.value

    def extend(self, seq: int, n_tokens: int):
        slots = torch.empty((max(n_tokens, 0),), dtype=torch.int64)
        src, dst = ctypes.c_int32(), ctypes.c_int32()
        _check(lib.aqmb_pages_extend(self.handle, seq, n_tokens, slots.data_ptr(), ctypes.byref(src),
                                     ctypes.byref(dst)), "aqmb_pages_extend")
        return slots, [(src.value, dst.value)] if src.value >= 0 else []

    def free(self, seq: int) -> None:
        _check(lib.aqmb_pages_free(self.handle, seq), "aqmb_pages_free")

    def compact(self):
        room = max(1, self.n_pages // 2)
        src, dst, n = (ctypes.c_int32 * room)(), (ctypes.c_int32 * room)(), ctypes.c_int()
        _check(lib.aqmb_pages_compact(self.handle, src, dst, ctypes.byref(n)), "aqmb_pages_compact")
        return list(zip(src[:n.value], dst[:n.value]))

    def _sizes(self, seq: int):
        n, length = ctypes.c_int(), ctypes.c_int()
        _check(lib.aqmb_pages_table(self.handle, seq, None, 0, ctypes.byref(n), ctypes.byref(length)),
               "aqmb_pages_table")
        return n.value, length.value

    def length(self, seq: int) -> int:
        return self._sizes(seq)[1]

    def table(self, seq: int):
        n, length = ctypes.c_int(), ctypes.c_int()
        pages = torch.empty((self._sizes(seq)[0],), dtype=torch.int32)
        if pages.numel():
            _check(lib.aqmb_pages_table(self.handle, seq, pages.data_ptr(), pages.numel(), ctypes.byref(n),
                                        ctypes.byref(length)), "aqmb_pages_table")
        return pages

    def counts(self):
        """(free pages, live sequences)"""
        f, s = ctypes.c_int(), ctypes.c_int()
        _check(lib.aqmb_pages_counts(self.handle, ctypes.byref(f), ctypes.byref(s)), "aqmb_pages_counts")
        return f.value, s.value

    def close(self):
        if self.handle:
            _check(lib.aqmb_pages_destroy(self.handle), "aqmb_pages_destroy")
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
