"""Rows in 8 bits, MS-RMSNorm into 8 bits and linear layers on them, in float64.

Test infrastructure only (see the package docstring).

Rows: a = max(max |t|, 2^-100), r = 127 / a held in 32 bits, q = t r rounded half to even
(t r of a row held in at most 32 bits is exact in float64: 24 + 24 bits), scale = a / 127. A
row that is not finite has q = 0 and scale NaN.

The gradient of a linear layer's input: dy w_scale is held in 32 bits before its rows are
brought to 8 bits.
"""

import numpy as np

from .dtypes import round_to_dtype


def _f32(a):
    return np.asarray(a, dtype=np.float64).astype(np.float32).astype(np.float64)


def rows(t):
    """(q as float64 whole numbers, scale) of the rows of t."""
    t = np.asarray(t, dtype=np.float64)
    q, a = _quantised(t)
    return q, a / 127.0


def _quantised(t):
    with np.errstate(invalid="ignore"):
        a = np.maximum(np.abs(t).max(axis=1), 2.0 ** -100)
        finite = np.isfinite(t).all(axis=1)
        a = np.where(finite, a, np.nan)
        r = _f32(127.0 / a)
        q = np.where(finite[:, None], np.rint(t * r[:, None]), 0.0)
    return q, a


def values(q, scale):
    return np.asarray(q, dtype=np.float64) * np.asarray(scale, dtype=np.float64)[:, None]


def msrms_fwd(x, res, eps, dtype):
    """(q, scale, rstd, s) of x, or of x + res rounded to dtype."""
    x = np.asarray(x, dtype=np.float64)
    s = x if res is None else round_to_dtype(x + np.asarray(res, dtype=np.float64), dtype)
    q, a = _quantised(s)
    rstd = 1.0 / np.sqrt((s * s).sum(axis=1) / s.shape[1] + float(eps))
    return q, a * rstd / 127.0, rstd, s


def msrms_bwd(dz, q, scale, rstd, ds=None):
    z, dz = values(q, scale), np.asarray(dz, dtype=np.float64)
    along = (z * dz).sum(axis=1, keepdims=True) / z.shape[1]
    dx = np.asarray(rstd, dtype=np.float64)[:, None] * (dz - z * along)
    return dx if ds is None else dx + np.asarray(ds, dtype=np.float64)


def linear_fwd(q, scale, w, w_scale, bias=None):
    y = values(q, scale) @ values(w, w_scale).T
    return y if bias is None else y + np.asarray(bias, dtype=np.float64)


def linear_bwd(dy, w, w_scale):
    p, scale = rows(_f32(np.asarray(dy, dtype=np.float64) * np.asarray(w_scale, dtype=np.float64)))
    return (p @ np.asarray(w, dtype=np.float64)) * scale[:, None]
