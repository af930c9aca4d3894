"""Pins of the 8-bit oracle against things other than itself."""

from fractions import Fraction

import numpy as np
import pytest

import oracle
from oracle import q8


def _f32(shape, seed, scale=1.0):
    return (np.random.default_rng(seed).standard_normal(shape) * scale).astype(np.float32)


def test_rows_by_exact_fractions():
    """q by brute force over the whole numbers, in rational arithmetic."""
    t = _f32((5, 37), 1)
    t[0, 3] = 0.0
    t[1] = np.float32(0.5)              # every value is the largest: 127
    t[2, :2] = [1.0, 0.5]               # 63.5 when 1 is the largest: a tie, to the even 64
    t[2, 2:] = np.clip(t[2, 2:], -0.9, 0.9)
    q, scale = q8.rows(t.astype(np.float64))
    for i in range(t.shape[0]):
        a = max(abs(Fraction(float(v))) for v in t[i])
        r = Fraction(float(np.float32(float(Fraction(127) / a))))
        for j in range(t.shape[1]):
            v = Fraction(float(t[i, j])) * r
            best = min(range(-128, 129), key=lambda c: (abs(v - c), c % 2))
            assert q[i, j] == best
        assert abs(scale[i] - float(a / 127)) <= 1e-15 * float(a)
    assert q[2, 0] == 127 and q[2, 1] == 64
    assert (q[1] == 127).all()


def test_rows_that_hold_nothing_or_too_much():
    t = np.zeros((4, 8))
    t[1, 2], t[2, 5], t[3, 0] = np.inf, np.nan, 2.0 ** -130
    q, scale = q8.rows(t)
    assert (q == 0).all()
    assert scale[0] == scale[3] == 2.0 ** -100 / 127 and np.isnan(scale[1:3]).all()


def test_norm_against_the_norm():
    """The values are those of MS-RMSNorm up to half a scale, the statistic its own."""
    x, res = _f32((6, 50), 2), _f32((6, 50), 3)
    q, scale, rstd, s = q8.msrms_fwd(x, res, 1e-5, "fp32")
    z, r = oracle.msrms_fwd((x + res).astype(np.float64), 1e-5)
    assert np.abs(r - rstd).max() <= 1e-12
    # half a step, and what the rounding of r to 32 bits moves: 127 * 2^-24 steps
    assert (np.abs(q8.values(q, scale) - z) <= scale[:, None] * (0.5 + 127 * 2.0 ** -23)).all()


def test_norm_gradient_by_differences():
    """At the exact z instead of its 8-bit form the backward is the norm's own derivative."""
    x, dz = _f32((3, 20), 4).astype(np.float64), _f32((3, 20), 5).astype(np.float64)
    eps, h = 1e-5, 1e-6
    z, rstd = oracle.msrms_fwd(x, eps)
    dx = q8.msrms_bwd(dz, z, np.ones(3), rstd)
    for j in range(20):
        step = np.zeros_like(x)
        step[:, j] = h
        diff = ((oracle.msrms_fwd(x + step, eps)[0] - oracle.msrms_fwd(x - step, eps)[0]) * dz).sum(axis=1) / (2 * h)
        assert np.abs(diff - dx[:, j]).max() <= 1e-7   # h^2 and 1e-16 / h
    ds = _f32((3, 20), 6)
    assert np.array_equal(q8.msrms_bwd(dz, z, np.ones(3), rstd, ds), dx + ds)


def test_linear_and_its_gradient():
    rng = np.random.default_rng(7)
    w, ws = rng.integers(-127, 128, (9, 13)), np.abs(_f32(9, 8)).astype(np.float64)
    q, qs = rng.integers(-127, 128, (4, 13)), np.abs(_f32(4, 9)).astype(np.float64)
    b = _f32(9, 10).astype(np.float64)
    y = q8.linear_fwd(q, qs, w, ws, b)
    for i in range(4):
        for j in range(9):
            want = sum(int(q[i, k]) * int(w[j, k]) for k in range(13)) * qs[i] * ws[j] + b[j]
            assert abs(y[i, j] - want) <= 1e-9
    # the layer is linear: its input's gradient is dy W, up to half a step of p per channel
    dy = _f32((4, 9), 11)
    dx = q8.linear_bwd(dy, w, ws)
    want = dy.astype(np.float64) @ (w * ws[:, None])
    step = np.abs(dy * ws).max(axis=1) / 127
    room = (0.5 + 1e-4) * step[:, None] * np.abs(w).sum(axis=0)[None, :]
    assert (np.abs(dx - want) <= room).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_the_sum_is_rounded_to_the_storage_type(dtype):
    x, res = _f32((2, 30), 12), _f32((2, 30), 13)
    s = q8.msrms_fwd(x, res, 1e-5, dtype)[3]
    assert np.array_equal(s, oracle.round_to_dtype(x.astype(np.float64) + res, dtype))
