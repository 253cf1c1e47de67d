"""Microscaled 4-bit matrices (MX4) and the products at them (float64 NumPy).

Test infrastructure only; see the package docstring.  Written from the format's
definition: a value is step * 2^(b - 127), the steps 0, 1/2, 1, 3/2, 2, 3, 4, 6 with a
sign, one exponent b per 32 columns.
"""
from __future__ import annotations

import numpy as np

from .numerics import silu

STEPS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK, GROUP = 32, 256


def exponent_of(amax):
    """Biased exponent b of the scale for a block's largest magnitude (255: not finite)."""
    amax = np.asarray(amax, np.float64)
    _, e = np.frexp(np.where(np.isfinite(amax), amax, 1.0))   # amax = m 2^e, m in [1/2, 1)
    b = np.where(amax > 0, np.maximum(e - 1 + 127 - 2, 0), 0)
    return np.where(np.isfinite(amax), b, 255).astype(np.int64)


def nearest_code(q):
    """Code of the step nearest to q, ties to the even code, the sign in bit 3."""
    a = np.minimum(np.abs(q), 6.0)
    dist = np.abs(a[..., None] - STEPS)
    lo = np.argmin(dist, axis=-1)                     # the first of two equally near
    tie = np.take_along_axis(dist, np.minimum(lo + 1, 7)[..., None], -1)[..., 0] == \
        np.take_along_axis(dist, lo[..., None], -1)[..., 0]
    code = np.where(tie & (lo < 7) & (lo % 2 == 1), lo + 1, lo)
    return code + 8 * np.signbit(q)


def quantize(x):
    """x [..., R, C] -> codes [..., R, C / 2] uint8, scale [..., ceil(C / 256), R, 8] uint8."""
    x = np.asarray(x, np.float64)
    C = x.shape[-1]
    v = x.reshape(x.shape[:-1] + (C // BLOCK, BLOCK))
    amax = np.where(np.isfinite(v).all(-1), np.abs(np.nan_to_num(v)).max(-1), np.inf)
    b = exponent_of(amax)
    ok = b[..., None] != 255
    code = np.where(ok, nearest_code(np.ldexp(np.where(ok, v, 0.0), 127 - b[..., None])), 0)
    code = code.reshape(x.shape).astype(np.uint8)
    b = np.concatenate([b, np.zeros(b.shape[:-1] + (-b.shape[-1] % 8,), b.dtype)], -1)
    b = b.reshape(b.shape[:-1] + (-1, 8))
    return code[..., 0::2] | code[..., 1::2] << 4, \
        np.ascontiguousarray(np.moveaxis(b, -2, -3)).astype(np.uint8)


def dequantize(codes, scale):
    """The values [..., R, C] in float64 (NaN where the scale is 255)."""
    codes, scale = np.asarray(codes), np.asarray(scale).astype(np.int64)
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))
    v = np.where(c & 8, -1.0, 1.0) * STEPS[c & 7]
    b = np.moveaxis(scale, -3, -2)
    b = b.reshape(b.shape[:-2] + (-1,))[..., :v.shape[-1] // BLOCK]
    s = np.where(b == 255, np.nan, np.ldexp(1.0, b - 127))
    return v * np.repeat(s, BLOCK, axis=-1)


def grouped_product(x_rows, w, offsets, expert_map=None):
    """(out [R, N], sum of magnitudes [R, N]): x_rows[r] times w[slot(e)]'s rows; NaN in
    rows of experts without a slot and outside every expert."""
    R, N = x_rows.shape[0], w.shape[1]
    out, mag = np.full((R, N), np.nan), np.full((R, N), np.nan)
    for e in range(len(offsets) - 1):
        slot = e if expert_map is None else expert_map[e]
        rows = slice(offsets[e], offsets[e + 1])
        if slot >= 0:
            out[rows] = x_rows[rows] @ w[slot].T
            mag[rows] = np.abs(x_rows[rows]) @ np.abs(w[slot]).T
    return out, mag


def swiglu(a):
    f = a.shape[-1] // 2
    return silu(a[..., :f]) * a[..., f:]
