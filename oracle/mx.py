"""Oracle of the microscaled 4-bit format (test infrastructure only).

TEST INFRASTRUCTURE ONLY: used by the tests; the product path never imports it.

A block of 32 values shares 2^e; an element is the nearest of sixteen values,
found by comparing distances (exact in float64: a value has at most 24
significand bits and the levels 3), of two equally near the one with the even
code.
"""

from __future__ import annotations

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def scale_stride(K):
    return -(-(K // 32) // 8) * 8


def quantize(x):
    """float64 [R, K] -> packed elements [R, K / 2], scale bytes [R, scale_stride(K)]."""
    x = np.asarray(x, dtype=np.float64)
    R, K = x.shape
    v = x.reshape(R, K // 32, 32)
    bad = ~np.isfinite(v).all(axis=2)
    top = np.where(bad, 0.0, np.abs(np.where(np.isfinite(v), v, 0.0)).max(axis=2))
    # frexp: top = f * 2^n with f in [0.5, 1), so floor(log2 top) = n - 1
    n = np.frexp(top)[1]
    e = np.where(top > 0, np.maximum(n - 1 - 2, -127), -127)
    y = np.ldexp(np.abs(np.where(bad[:, :, None], 0.0, v)), -e[:, :, None])
    dist = np.abs(y[..., None] - LEVELS)
    code = np.argmin(dist, axis=-1)  # the lower of two equally near
    up = np.minimum(code + 1, 7)
    tie = (up > code) & (np.take_along_axis(dist, up[..., None], -1)[..., 0] == dist.min(axis=-1))
    code = np.where(tie & (code % 2 == 1), up, code)
    code = code + 8 * np.signbit(np.where(bad[:, :, None], 0.0, v))
    code = code.reshape(R, K).astype(np.uint8)
    s = np.zeros((R, scale_stride(K)), dtype=np.uint8)
    s[:, :K // 32] = np.where(bad, 255, e + 127)
    return code[:, 0::2] | (code[:, 1::2] << 4), s


def values(q, s, K):
    """packed elements and scale bytes -> float64 [R, K], NaN where the scale byte is 255."""
    R = q.shape[0]
    code = np.empty((R, K), dtype=np.int64)
    code[:, 0::2], code[:, 1::2] = q & 15, q >> 4
    v = np.where(code >= 8, -1.0, 1.0) * LEVELS[code & 7]
    e = s[:, :K // 32].astype(np.int64)
    by = np.where(e == 255, np.nan, np.ldexp(1.0, np.where(e == 255, 0, e - 127)))
    return (v.reshape(R, K // 32, 32) * by[:, :, None]).reshape(R, K)
