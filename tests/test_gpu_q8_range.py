"""Rows of every size through MS-RMSNorm into 8 bits and back.

A finite row stands for s rstd whatever its size, also where its squares add up to more than
fp32 holds or, with an eps as small, are less than it holds; and so does the backward's sum of
q dz where it is more. The bounds are those of test_gpu_q8_rows.py (chains of p / 64 + 24 additions, then the roundings counted there: scaling by a power of two
rounds nothing), and half a step of the smallest numbers, 2^-150, where rstd is one of them.
"""

import numpy as np
import pytest
import torch

import paper_2406_16282_amd as lmbp
from oracle import q8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
# the register form with 1, 2, 4, 8 and 16 waves to a row, rows at any address, and a block per row
COLS = [1, 40, 768, 1025, 2049, 4096, 12345, 13824, 30011, 70000, 140001]
SIZES = [1.0, 2.0 ** 60, 2.0 ** 64, 2.0 ** 100, 2.0 ** 122, 2.0 ** -40, 2.0 ** -71, 0.0]


def n64(t):
    return t.detach().double().cpu().numpy()


def draw(rows, cols, dtype, seed, sizes):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g).clamp_(-8, 8)
    x *= torch.tensor([sizes[i % len(sizes)] for i in range(rows)])[:, None]
    return x.to(TYPES[dtype]).to(DEV)


def rows_of_every_size(cols, dtype, seed):
    x = draw(13, cols, dtype, seed, SIZES)
    x[8:] = draw(5, cols, dtype, seed + 1, [1.0])
    x[8, cols // 2] = 2.0 ** 80          # one value far above the rest of its row
    x[9, cols - 1] = -2.0 ** 127
    x[10, 0] = 2.0 ** 66
    x[11] = 2.0 ** 127                   # all of them as large as they come
    x[12, : (cols + 1) // 2] *= 2.0 ** -60
    return x


@pytest.mark.parametrize("eps", [1e-5, 1e-30, 1e30, 1e-44])
@pytest.mark.parametrize("with_res", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols", COLS)
def test_norm(cols, dtype, with_res, eps):
    print(f"[q8] range {cols} {dtype} res {with_res} eps {eps}", flush=True)
    x = rows_of_every_size(cols, dtype, 1)
    res = draw(13, cols, dtype, 3, [1.0, 2.0 ** 58, 2.0 ** 30, 2.0 ** 99]) if with_res else None
    q, scale, rstd, *s = lmbp.msrms_q8_fwd(x, eps, res)
    torch.cuda.synchronize()
    q_o, sc_o, r_o, s_o = q8.msrms_fwd(n64(x), None if res is None else n64(res), float(np.float32(eps)), dtype)
    assert np.isfinite(s_o).all()
    if with_res:
        assert np.array_equal(n64(s[0]), s_o)
    assert np.array_equal(n64(q), q_o)
    c = cols / 64 + 24
    assert (np.abs(n64(rstd) - r_o) <= 1.01 * U * (c / 2 + 4) * r_o + 2.0 ** -149).all()
    assert (np.abs(n64(scale) - sc_o) <= 1.01 * U * (c / 2 + 6) * sc_o + 2.0 ** -149).all()


@pytest.mark.parametrize("dt_dz,dtype", [("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("cols", COLS)
def test_norm_backward(cols, dt_dz, dtype):
    x = draw(13, cols, dtype, 5, [1.0, 2.0 ** 3, 2.0 ** 70, 2.0 ** -3, 2.0 ** 110])
    q, scale, rstd = lmbp.msrms_q8_fwd(x, 1e-5)
    dz = draw(13, cols, dt_dz, 6, [1e-3, 2.0 ** 121, 2.0 ** 118, 2.0 ** -60, 2.0 ** 100, 2.0 ** 122])
    ds = draw(13, cols, dtype, 7, [1e-3, 2.0 ** 100])
    for more in (None, ds):
        dx = lmbp.msrms_q8_bwd(dz, q, scale, rstd, more, dtype=TYPES[dtype])
        torch.cuda.synchronize()
        dx_o = q8.msrms_bwd(n64(dz), n64(q), n64(scale), n64(rstd), None if more is None else n64(more))
        c = cols / 64 + 24
        g, w, sc, rs = n64(dz), n64(q), n64(scale)[:, None], n64(rstd)[:, None]
        most = np.abs(w) * sc * sc / cols * np.abs(w * g).sum(axis=1, keepdims=True)
        # what passes the largest number of the type (2^128) is none of this test's: no value here does
        assert (np.abs(dx_o) < 2.0 ** 127).all() and (np.abs(g) + most < 2.0 ** 127).all()
        room = rs * most * (c + 4) * U + 3 * U * (rs * (np.abs(g) + most) + np.abs(dx_o))
        room = 1.01 * (room + torch.finfo(TYPES[dtype]).eps / 2 * np.abs(dx_o)) + 2.0 ** -133
        assert (np.abs(n64(dx) - dx_o) <= room).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols", COLS)
def test_in_place(cols, dtype):
    """The sum in place of x or of the residual, dx in place of dz or of ds, where rows are added up again."""
    x, res = rows_of_every_size(cols, dtype, 1), draw(13, cols, dtype, 3, [1.0, 2.0 ** 58, 2.0 ** 30, 2.0 ** 99])
    want = lmbp.msrms_q8_fwd(x, 1e-5, res)
    for into in ("x", "res"):
        a, b = x.clone(), res.clone()
        got = lmbp.msrms_q8_fwd(a, 1e-5, b, s=a if into == "x" else b)
        assert all(torch.equal(g, w) for g, w in zip(got, want))
    q, scale, rstd, _ = want
    dz, ds = draw(13, cols, dtype, 6, [1e-3, 2.0 ** 121, 2.0 ** 118]), draw(13, cols, dtype, 7, [1e-3, 2.0 ** 100])
    dx = lmbp.msrms_q8_bwd(dz, q, scale, rstd, ds)
    a, b = dz.clone(), ds.clone()
    assert torch.equal(lmbp.msrms_q8_bwd(a, q, scale, rstd, ds, dx=a).view(torch.uint8), dx.view(torch.uint8))
    assert torch.equal(lmbp.msrms_q8_bwd(dz, q, scale, rstd, b, dx=b).view(torch.uint8), dx.view(torch.uint8))


@pytest.mark.parametrize("cols", [40, 1025, 4096, 13824, 30011, 140001])
def test_rows_that_are_not_finite_beside_large_ones(cols):
    """An infinity or a NaN stays in its row; the rows beside it are as without it."""
    x = rows_of_every_size(cols, "fp32", 1)
    dz = draw(13, cols, "fp32", 6, [1e-3, 2.0 ** 121, 2.0 ** 118])
    q, scale, rstd = lmbp.msrms_q8_fwd(x, 1e-5)
    dx = lmbp.msrms_q8_bwd(dz, q, scale, rstd)
    bad, keep = [1, 4, 9], [i for i in range(13) if i not in (1, 4, 9)]
    y, dy = x.clone(), dz.clone()
    for row, value in zip(bad, (float("inf"), float("nan"), -float("inf"))):
        y[row, cols // 3] = value
        dy[row, cols // 2] = value
    q1, scale1, rstd1 = lmbp.msrms_q8_fwd(y, 1e-5)
    assert (q1[bad] == 0).all() and scale1[bad].isnan().all()
    for a, b in zip((q1, scale1, rstd1), (q, scale, rstd)):
        assert torch.equal(a[keep], b[keep])
    dx1 = lmbp.msrms_q8_bwd(dy, q, scale, rstd)
    assert torch.equal(dx1[keep], dx[keep]) and not dx1[bad].isfinite().all(dim=1).any()
