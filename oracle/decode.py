"""Definitions in 64 bits of the operators between the layers of a decode step.

Root-mean-square norm with the residual's addition, scaling to 8 bits, products with 4-bit weights,
attention of one token over a paged cache; rotary positions, low-rank adapters and log probabilities. Plain NumPy loops and sums; inputs are fp64 arrays that
hold the exact values of the stored formats. The definitions are those of ``include/aqmb.h``;
the paper does not treat these operators (parity unpinned by it; closed forms pin them in
``tests/test_oracle_decode.py``).
"""
from __future__ import annotations

import numpy as np

LARGEST = {"f8": 448.0, "i8": 127.0}
FLOOR = 2.0 ** -100


def rms_norm(x, residual, weight, offset, eps):
    """(h, v): the sum with the residual (None: x alone) and the scaled norm, both before any rounding."""
    h = x if residual is None else x + residual
    rms = np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    return h, h / rms * (weight + offset)[None, :]


def scaled(v, group, largest):
    """(grid, scales): v [rows][cols] as multiples of its groups' scales, before rounding to 8 bits."""
    rows, cols = v.shape
    group = group or cols
    grid, scales = np.empty_like(v), np.empty((rows, -(-cols // group)))
    for j in range(scales.shape[1]):
        part = v[:, j * group:(j + 1) * group]
        a = np.maximum(np.abs(part).max(axis=1), FLOOR)
        scales[:, j] = a / largest
        grid[:, j * group:(j + 1) * group] = part * (largest / a)[:, None]
    return grid, scales


def e4m3_step(t):
    """Spacing of e4m3 at |t| (largest 448, subnormals in steps of 2^-9)."""
    a = np.maximum(np.abs(t), 2.0 ** -6)
    return 2.0 ** (np.floor(np.log2(a)) - 3)


def e4m3_decode(bits):
    """e4m3 bit patterns (uint8) -> fp64."""
    b = np.asarray(bits, dtype=np.int64)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((e == 15) & (m == 7), np.nan, v)
    return np.where(b & 128, -v, v)


def nibbles(weights, d_in):
    """[d_out][ceil(d_in/2)] bytes -> [d_out][d_in] integers 0..15, low nibble first."""
    w = np.asarray(weights, dtype=np.int64)
    q = np.empty((w.shape[0], 2 * w.shape[1]), dtype=np.int64)
    q[:, 0::2], q[:, 1::2] = w & 15, w >> 4
    return q[:, :d_in]


def w4_weights(weights, scales, zeros, d_in, group):
    """The dense matrix [d_out][d_in]: scale (q - zero), zero 8 where there is none."""
    per = np.arange(d_in) // group
    z = 8.0 if zeros is None else np.asarray(zeros, dtype=np.float64)[:, per]
    return (nibbles(weights, d_in) - z) * scales[:, per]


def attend(q, keys, values, scale):
    """One query [dim] over keys, values [n][dim]: (out [dim], log of the denominator). n may be 0."""
    if len(keys) == 0:
        return np.zeros(values.shape[1]), -np.inf
    s = keys @ q * scale
    m = s.max()
    p = np.exp(s - m)
    return p @ values / p.sum(), m + np.log(p.sum())


def paged_attention(q, k, v, table, lengths, scale, window=0, layout="head"):
    """q [n][heads][dim]; k, v [pages][kv][size][dim] ("head") or [pages][size][kv][dim] ("slot"), already
    multiplied by their scales; table: a page per row entry, entries outside the cache are skipped."""
    n, heads, dim = q.shape
    if layout == "slot":
        k, v = k.transpose(0, 2, 1, 3), v.transpose(0, 2, 1, 3)
    kv, size = k.shape[1], k.shape[2]
    out, lse = np.zeros((n, heads, dim)), np.full((n, heads), -np.inf)
    for i in range(n):
        pos = range(max(0, lengths[i] - window) if window else 0, lengths[i])
        where = [(table[i][t // size], t % size) for t in pos if 0 <= table[i][t // size] < k.shape[0]]
        page, slot = [w[0] for w in where], [w[1] for w in where]
        for h in range(heads):
            g = h // (heads // kv)
            out[i, h], lse[i, h] = attend(q[i, h], k[page, g, slot] if where else np.zeros((0, dim)),
                                          v[page, g, slot] if where else np.zeros((0, dim)), scale)
    return out, lse


def rotary(x, angles, half, amplitude=1.0):
    """x [n][heads][dim] with its first 2 * angles.shape[1] values turned in pairs by angles [n][pairs]: values i and
    i + pairs (half) or 2 i and 2 i + 1."""
    n, y = angles.shape[1], np.array(x, dtype=np.float64)
    for i in range(n):
        a, b = (i, i + n) if half else (2 * i, 2 * i + 1)
        c, s = np.cos(angles[:, i])[:, None], np.sin(angles[:, i])[:, None]
        y[..., a] = amplitude * (x[..., a] * c - x[..., b] * s)
        y[..., b] = amplitude * (x[..., b] * c + x[..., a] * s)
    return y


def adapted(x, index, a, b, scales, ranks):
    """scales[n] * b[n] (a[n] x) for every row of x with n = index[row], 0 where there is no such adapter."""
    y = np.zeros((x.shape[0], b.shape[1]))
    for i, n in enumerate(index):
        if 0 <= n < a.shape[0]:
            r = min(max(int(ranks[n]), 0), a.shape[1])
            y[i] = scales[n] * (b[n, :, :r] @ (a[n, :r] @ x[i]))
    return y


def log_probs(z):
    """(log p, log sum exp, entropy) of one row z; -infinity weighs nothing, NaN or +infinity makes all of it NaN."""
    if np.isnan(z).any() or (z == np.inf).any():
        return np.full_like(z, np.nan), np.nan, np.nan
    top = z.max()
    if top == -np.inf:
        return z, -np.inf, 0.0
    s = np.log(np.exp(z - top).sum())
    lp = z - top - s                  # of the sum's logarithm nothing is left in 64 bits beside a top of 1e38
    return lp, top + s, -sum(np.exp(v) * v for v in lp if v > -np.inf)
