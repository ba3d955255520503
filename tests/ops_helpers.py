"""Shared by the GPU tests of the operators between the layers: exact values of device tensors and
the spacing of a format, in fp64."""
import numpy as np
import torch

from oracle import decode, formats

U = 2.0 ** -24                      # half the spacing of binary32 at one
FMT = {torch.float16: "f16", torch.bfloat16: "bf16", torch.float32: "f32"}


def values(t):
    """A tensor of any of the operators' types -> exact fp64 NumPy values."""
    t = t.detach().contiguous().cpu()
    if t.dtype == torch.float8_e4m3fn:
        return decode.e4m3_decode(t.view(torch.uint8).numpy())
    if t.dtype in (torch.float16, torch.bfloat16):
        b = t.view(torch.int16).numpy().view(np.uint16)
        return formats.f16_bits_to_f64(b) if t.dtype == torch.float16 else formats.bf16_bits_to_f64(b)
    return t.numpy().astype(np.float64)


def half_ulp(ref, dtype):
    return 0.5 * formats.ulp_of(ref, FMT[dtype])


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)
