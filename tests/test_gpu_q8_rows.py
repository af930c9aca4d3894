"""GPU parity of rows in 8 bits and of MS-RMSNorm into 8 bits against the 64-bit oracle.

Whole numbers are compared exactly. Bounds of the floating outputs, with u = 2^-24 (half a step
of fp32, relative) and h half a step of the storage type:

* scale of plain rows: one division, u;
* rstd: a sum of p squares in chains of at most c = p / 64 + 24 additions, each u of a partial
  sum of positive terms, halved by the root; the mean, eps and rsqrt (two roundings at most)
  another 4 u;
* scale of the norm: rstd's and two more;
* dx = rs (dz - q b) + ds, b = sc^2 p^-1 sum(q dz): the sum is off by c u sum |q dz|, b by 4 u of
  itself more, then three roundings of the terms and one to the storage type.
"""

import ctypes

import numpy as np
import pytest
import torch

import paper_2406_16282_amd as lmbp
from oracle import q8
from paper_2406_16282_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
EPS = 1e-5
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SHAPES = [(1, 1), (3, 1), (5, 2), (1, 8), (2, 33), (1, 4096), (64, 768), (7, 1023), (33, 1025), (130, 96), (4, 5120),
          (3, 8191), (2, 11008), (3, 13824), (5, 12345), (2, 16392), (2, 30011), (1, 40000), (2, 65536), (1, 131080)]


def half(dtype):
    return torch.finfo(TYPES[dtype]).eps / 2


def n64(t):
    return t.detach().double().cpu().numpy()


def draw(rows, cols, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, cols, generator=g) * scale).to(TYPES[dtype]).to(DEV)


def stream_rows(rows, cols, dtype, seed):
    """Rows of sizes from tiny to large, zeros, one large value and ties among them."""
    x = draw(rows, cols, dtype, seed)
    size = torch.tensor([1.0, 2.0 ** -60, 2.0 ** 40, 0.0, 2.0 ** -110, 3.7], device=DEV)
    x = x * size[torch.arange(rows, device=DEV) % 6].to(x.dtype)[:, None]
    if rows > 6 and cols > 2:
        x[6] = 0.5
        x[6, cols // 2] = 1.0     # every other value is a tie: 63.5 goes to 64
    return x.contiguous()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_rows_and_values(rows, cols, dtype):
    print(f"[q8] rows {rows} x {cols} {dtype}", flush=True)
    x = stream_rows(rows, cols, dtype, rows * cols)
    q, scale = lmbp.q8_rows(x)
    v = lmbp.q8_values(q, scale, TYPES[dtype])
    torch.cuda.synchronize()
    q_o, s_o = q8.rows(n64(x))
    assert q.shape == x.shape and scale.shape == (rows,)
    assert np.array_equal(n64(q), q_o)
    assert (np.abs(n64(scale) - s_o) <= 1.01 * U * s_o).all()
    v_o = q8.values(q_o, n64(scale))
    assert (np.abs(n64(v) - v_o) <= 1.01 * (U + half(dtype)) * np.abs(v_o) + 2.0 ** -133).all()
    # the values are the rows again, up to half a scale and the rounding of r and of v
    assert (np.abs(v_o - n64(x)) <= (0.5 + 127 * 4 * U) * s_o[:, None]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols", [1, 7, 768, 1025, 13824, 70000])
def test_rows_that_are_not_finite(cols, dtype):
    x = draw(6, cols, dtype, 3)
    for row, (col, bad) in enumerate([(0, np.inf), (cols - 1, -np.inf), (cols // 2, np.nan)]):
        x[row, col] = float(bad)
    if dtype == "fp32":   # a NaN whose low bits are not zero
        x.view(torch.int32)[2, cols // 2] = 0x7F812345
    x[3] = 0.0
    q, scale = lmbp.q8_rows(x)
    qn, sn, rstd = lmbp.msrms_q8_fwd(x, EPS)
    torch.cuda.synchronize()
    for got, s in ((q, scale), (qn, sn)):
        assert (got[:4] == 0).all() and s[:3].isnan().all() and s[3:].isfinite().all()
        assert np.array_equal(n64(got[4:]), q8.rows(n64(x[4:]))[0])
    assert lmbp.q8_values(q, scale)[:3].isnan().all()
    dx = lmbp.msrms_q8_bwd(torch.ones_like(x), qn, sn, rstd)
    assert dx[:3].isnan().all() and dx[3:].isfinite().all()


def norm_bounds(x, s_o, cols):
    c = cols / 64 + 24
    return 1.01 * U * (c / 2 + 4), 1.01 * U * (c / 2 + 6)


def bwd_bound(dz, q, scale, rstd, dx, cols, dtype):
    c = cols / 64 + 24
    dz, q, sc, rs = n64(dz), n64(q), n64(scale)[:, None], n64(rstd)[:, None]
    most = np.abs(q) * sc * sc / cols * np.abs(q * dz).sum(axis=1, keepdims=True)
    return 1.01 * (rs * most * (c + 4) * U + 3 * U * (rs * (np.abs(dz) + most) + np.abs(dx)) + half(dtype) * np.abs(dx)) + 2.0 ** -133


@pytest.mark.parametrize("with_res", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm(rows, cols, dtype, with_res):
    print(f"[q8] norm {rows} x {cols} {dtype} res {with_res}", flush=True)
    x = draw(rows, cols, dtype, 1)
    if rows > 2:
        x[1] = 0.0
    res = draw(rows, cols, dtype, 2, 3.0) if with_res else None
    if rows > 2 and with_res:
        res[1] = 0.0
        res[2] = -x[2]      # a sum of nothing
    dz, ds = draw(rows, cols, dtype, 4, 1e-3), draw(rows, cols, dtype, 5, 1e-3) if with_res else None
    q, scale, rstd, *s = lmbp.msrms_q8_fwd(x, EPS, res)
    dx = lmbp.msrms_q8_bwd(dz, q, scale, rstd, ds)
    torch.cuda.synchronize()
    assert len(s) == int(with_res)
    eps32 = float(np.float32(EPS))
    q_o, sc_o, r_o, s_o = q8.msrms_fwd(n64(x), None if res is None else n64(res), eps32, dtype)
    if with_res:
        assert np.array_equal(n64(s[0]), s_o)
    assert np.array_equal(n64(q), q_o)
    rs_room, sc_room = norm_bounds(x, s_o, cols)
    assert (np.abs(n64(rstd) - r_o) <= rs_room * r_o).all()
    assert (np.abs(n64(scale) - sc_o) <= sc_room * sc_o).all()
    dx_o = q8.msrms_bwd(n64(dz), q_o, n64(scale), n64(rstd), None if ds is None else n64(ds))
    assert (np.abs(n64(dx) - dx_o) <= bwd_bound(dz, q, scale, rstd, dx_o, cols, dtype)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols", [(9, 64), (5, 1001), (3, 4096), (2, 70001)])
def test_sums_and_gradients_in_place(rows, cols, dtype):
    x, res = draw(rows, cols, dtype, 6), draw(rows, cols, dtype, 7)
    want = lmbp.msrms_q8_fwd(x, EPS, res)
    for target in ("x", "res", "both"):
        a, b = x.clone(), res.clone()
        if target == "both":    # one tensor as x, res and s
            b = a
            want_here = lmbp.msrms_q8_fwd(x, EPS, x.clone())
        else:
            want_here = want
        got = lmbp.msrms_q8_fwd(a, EPS, b, s=b if target == "res" else a)
        assert all(torch.equal(g, w) for g, w in zip(got, want_here))
    dz, ds = draw(rows, cols, dtype, 8), draw(rows, cols, dtype, 9)
    want = lmbp.msrms_q8_bwd(dz, *got[:3], ds)
    a, b = dz.clone(), ds.clone()
    assert torch.equal(lmbp.msrms_q8_bwd(a, *got[:3], ds, dx=a), want)
    assert torch.equal(lmbp.msrms_q8_bwd(dz, *got[:3], b, dx=b), want)
    assert torch.equal(lmbp.msrms_q8_bwd(b, *got[:3], b.clone()), lmbp.msrms_q8_bwd(b, *got[:3], b))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols,shift", [(5, 64, 1), (3, 1024, 3), (4, 1023, 1), (2, 13824, 1), (1, 66000, 2)])
def test_any_address_and_nothing_beside_the_rows(rows, cols, shift, dtype):
    """Every tensor `shift` elements behind an aligned address, between bands that stay as
    they were; the results are those of aligned tensors."""
    t, n = TYPES[dtype], rows * cols

    class Band:
        def __init__(self, count, dtype, fill=None):
            self.buf = torch.full((count + 64,), 85, dtype=dtype, device=DEV)
            self.t = self.buf[16 + shift:16 + shift + count]
            if fill is not None:
                self.t.copy_(fill.reshape(-1))

        @property
        def ptr(self):
            return ctypes.c_void_p(self.t.data_ptr())

        def whole(self):
            a, b = self.buf[:16 + shift], self.buf[16 + shift + self.t.numel():]
            return bool((a == 85).all() and (b == 85).all())

    x, res, dz = draw(rows, cols, dtype, 1), draw(rows, cols, dtype, 2), draw(rows, cols, dtype, 3)
    f32, i8 = torch.float32, torch.int8
    bx, bres, bdz, bs, bdx, bv = (Band(n, t, f) for f in (x, res, dz, None, None, None))
    bq, bsc, brs = Band(n, i8), Band(rows, f32), Band(rows, f32)
    L, dt = lmbp.lib(), B.BF16 if dtype == "bf16" else B.FP32
    st = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    want_q, want_sc, want_rs, want_s = lmbp.msrms_q8_fwd(x, EPS, res)
    assert L.msrms_q8_fwd(dt, rows, cols, EPS, bx.ptr, bres.ptr, bs.ptr, bq.ptr, bsc.ptr, brs.ptr, st) == B.OK
    assert torch.equal(bq.t.view(rows, cols), want_q) and torch.equal(bs.t.view(rows, cols), want_s)
    room = 2 * 1.01 * U * (cols / 128 + 18)     # two sums in orders of their own
    assert ((brs.t - want_rs).abs() <= room * want_rs).all() and ((bsc.t - want_sc).abs() <= room * want_sc).all()
    assert L.q8_values(dt, rows, cols, bq.ptr, bsc.ptr, bv.ptr, st) == B.OK
    assert torch.equal(bv.t.view(rows, cols), lmbp.q8_values(want_q, bsc.t.clone(), t))
    assert L.msrms_q8_bwd(dt, dt, rows, cols, bdz.ptr, bq.ptr, bsc.ptr, brs.ptr, bres.ptr, bdx.ptr, st) == B.OK
    dx_o = q8.msrms_bwd(n64(dz), n64(want_q), n64(bsc.t), n64(brs.t), n64(res))
    got = n64(bdx.t).reshape(rows, cols)
    assert (np.abs(got - dx_o) <= bwd_bound(dz, want_q, bsc.t, brs.t, dx_o, cols, dtype)).all()
    assert L.q8_rows(dt, rows, cols, bx.ptr, bq.ptr, bsc.ptr, st) == B.OK
    q, sc = lmbp.q8_rows(x)
    assert torch.equal(bq.t.view(rows, cols), q) and torch.equal(bsc.t, sc)
    torch.cuda.synchronize()
    assert all(b.whole() for b in (bx, bres, bdz, bs, bdx, bv, bq, bsc, brs))
    assert torch.equal(bx.t.view(rows, cols), x) and torch.equal(bdz.t.view(rows, cols), dz)


def test_more_than_2_31_values():
    """Rows far behind the 2^31st element and byte."""
    rows, cols = 270_000, 8192
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    at = [0, 131_071, 131_072, 262_143, 262_144, rows - 1]
    some = draw(len(at), cols, "bf16", 11)
    x[at] = some
    q, scale, rstd = lmbp.msrms_q8_fwd(x, EPS)
    want = lmbp.msrms_q8_fwd(some, EPS)
    for got, w in zip((q, scale, rstd), want):
        assert torch.equal(got[at], w)
    assert int((q[131_073:262_143] != 0).sum()) == 0
    x[at] = draw(len(at), cols, "bf16", 12)
    dx = lmbp.msrms_q8_bwd(x, q, scale, rstd)
    assert torch.equal(dx[at], lmbp.msrms_q8_bwd(x[at].contiguous(), *want))
    v = lmbp.q8_values(q, scale)
    assert torch.equal(v[at], lmbp.q8_values(want[0], want[1]))
    q2, scale2 = lmbp.q8_rows(x)
    q1, scale1 = lmbp.q8_rows(x[at].contiguous())
    assert torch.equal(q2[at], q1) and torch.equal(scale2[at], scale1)


def test_shapes_and_refusals():
    x = draw(6, 16, "bf16", 1)
    q, scale = lmbp.q8_rows(x.view(2, 3, 16))
    assert q.shape == (2, 3, 16) and scale.shape == (2, 3)
    q0, s0 = lmbp.q8_rows(x[:0])
    assert q0.shape == (0, 16) and s0.shape == (0,) and lmbp.q8_values(q0, s0).shape == (0, 16)
    assert lmbp.msrms_q8_bwd(x[:0], q0, s0, s0).shape == (0, 16)
    q, scale, rstd = lmbp.msrms_q8_fwd(x, EPS)
    cases = [
        (TypeError, lambda: lmbp.q8_rows(x.half())),
        (ValueError, lambda: lmbp.q8_rows(x.t())),
        (lmbp.LmbpError, lambda: lmbp.q8_rows(x[:, :0].contiguous())),
        (lmbp.LmbpError, lambda: lmbp.msrms_q8_fwd(x, 0.0)),
        (ValueError, lambda: lmbp.msrms_q8_fwd(x, EPS, x.float())),
        (ValueError, lambda: lmbp.msrms_q8_fwd(x, EPS, x.view(16, 6))),
        (ValueError, lambda: lmbp.msrms_q8_fwd(x, EPS, s=x)),
        (lmbp.LmbpError, lambda: lmbp.msrms_q8_fwd(x[:4], EPS, x[:4].clone(), s=x.view(-1)[8:72].view(4, 16))),
        (ValueError, lambda: lmbp.msrms_q8_bwd(x, q[:3], scale, rstd)),
        (ValueError, lambda: lmbp.msrms_q8_bwd(x, q.float(), scale, rstd)),
        (ValueError, lambda: lmbp.msrms_q8_bwd(x, q, scale[:3], rstd)),
        (ValueError, lambda: lmbp.msrms_q8_bwd(x, q, scale, rstd.double())),
        (ValueError, lambda: lmbp.msrms_q8_bwd(x, q, scale, rstd, x[:3])),
        (ValueError, lambda: lmbp.msrms_q8_bwd(x, q, scale, rstd, dx=x.float())),
        (TypeError, lambda: lmbp.msrms_q8_bwd(x, q, scale, rstd, dtype=torch.float16)),
        (lmbp.LmbpError, lambda: lmbp.msrms_q8_bwd(x, q, scale, rstd, x.float())),   # bf16 dz, fp32 dx
        (TypeError, lambda: lmbp.q8_values(q, scale, torch.float16)),
        (ValueError, lambda: lmbp.q8_values(q, scale[:2])),
        (ValueError, lambda: lmbp.q8_values(x, scale)),
    ]
    for error, call in cases:
        with pytest.raises(error):
            call()


@pytest.mark.parametrize("with_ds", [False, True])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm_backward_from_a_sum_in_fp32(rows, cols, with_ds):
    x = draw(rows, cols, "bf16", 1)
    q, scale, rstd = lmbp.msrms_q8_fwd(x, EPS)
    dz, ds = draw(rows, cols, "fp32", 4, 1e-3), draw(rows, cols, "bf16", 5, 1e-3) if with_ds else None
    dx = lmbp.msrms_q8_bwd(dz, q, scale, rstd, ds, dtype=torch.bfloat16)
    assert dx.dtype == torch.bfloat16
    dx_o = q8.msrms_bwd(n64(dz), n64(q), n64(scale), n64(rstd), None if ds is None else n64(ds))
    assert (np.abs(n64(dx) - dx_o) <= bwd_bound(dz, q, scale, rstd, dx_o, cols, "bf16")).all()
    if with_ds:   # in place of the gradient of the sum
        assert torch.equal(lmbp.msrms_q8_bwd(dz, q, scale, rstd, ds, dx=ds), dx)


def test_any_bytes_have_values():
    q = torch.arange(-128, 128, dtype=torch.int8, device=DEV).view(2, 128)
    scale = torch.tensor([0.5, -3.0], device=DEV)
    v = lmbp.q8_values(q, scale, torch.float32)
    assert torch.equal(v, q.float() * scale[:, None])
