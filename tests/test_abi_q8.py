"""The 8-bit entry points' checks on the host: nothing here reaches a GPU."""

import pytest
import torch

import paper_2406_16282_amd as lmbp
from paper_2406_16282_amd import binding as B
from paper_2406_16282_amd import nn as lnn

P = 0x7F0000000000   # fake device addresses: every call fails, or is a no-op, before a launch
MiB = 1 << 20


def at(i):
    return P + i * 64 * MiB


@pytest.fixture(scope="module")
def L():
    return lmbp.lib()


def test_q8_rows(L):
    def f(dt=B.BF16, rows=4, cols=32, x=at(0), q=at(1), scale=at(2)):
        return L.q8_rows(dt, rows, cols, x, q, scale, None)
    assert f(dt=5) == B.EDTYPE
    assert f(rows=-1) == f(cols=-1) == f(cols=0) == B.EINVAL
    assert f(rows=0, x=None, q=None, scale=None) == B.OK
    assert f(x=None) == f(q=None) == f(scale=None) == B.EINVAL
    assert f(x=at(0) + 1) == f(scale=at(2) + 2) == f(dt=B.FP32, x=at(0) + 2) == B.EINVAL
    assert f(rows=1 << 40, cols=1 << 40) == B.EINVAL
    assert f(q=at(0) + 255) == f(scale=at(0)) == f(scale=at(1) + 124) == B.EOVERLAP


def test_q8_values(L):
    def f(dt=B.BF16, rows=4, cols=32, q=at(0), scale=at(1), v=at(2)):
        return L.q8_values(dt, rows, cols, q, scale, v, None)
    assert f(dt=5) == B.EDTYPE
    assert f(rows=-1) == f(cols=-1) == f(cols=0) == B.EINVAL
    assert f(rows=0, q=None, scale=None, v=None) == B.OK
    assert f(q=None) == f(scale=None) == f(v=None) == B.EINVAL
    assert f(scale=at(1) + 1) == f(v=at(2) + 1) == B.EINVAL
    assert f(v=at(0) + 126) == f(v=at(1)) == B.EOVERLAP


def test_msrms_q8_fwd(L):
    def f(dt=B.BF16, rows=4, cols=32, eps=1e-5, x=at(0), res=at(1), s=at(2), q=at(3), scale=at(4), rstd=at(5)):
        return L.msrms_q8_fwd(dt, rows, cols, eps, x, res, s, q, scale, rstd, None)
    assert f(dt=5) == B.EDTYPE
    assert f(rows=-1) == f(cols=-1) == f(cols=0) == B.EINVAL
    assert f(rows=0, x=None, res=None, s=None, q=None, scale=None, rstd=None) == B.OK
    assert f(x=None) == f(q=None) == f(scale=None) == f(rstd=None) == B.EINVAL
    assert f(res=None) == f(s=None) == B.EINVAL          # both or none
    assert [f(eps=e) for e in (0.0, -1.0, float("inf"), float("nan"))] == [B.EINVAL] * 4
    assert f(x=at(0) + 1) == f(res=at(1) + 1) == f(s=at(2) + 1) == f(rstd=at(5) + 2) == B.EINVAL
    assert f(s=at(0) + 2) == f(s=at(1) + 2) == B.EOVERLAP       # not the exact pair
    assert f(q=at(0)) == f(q=at(1)) == f(q=at(2)) == f(scale=at(3)) == f(rstd=at(4)) == f(rstd=at(2)) == B.EOVERLAP


def test_msrms_q8_bwd(L):
    def f(dt=B.BF16, rows=4, cols=32, dz=at(0), q=at(1), scale=at(2), rstd=at(3), ds=at(4), dx=at(5), dt_dz=None):
        return L.msrms_q8_bwd(dt if dt_dz is None else dt_dz, dt, rows, cols, dz, q, scale, rstd, ds, dx, None)
    assert f(dt=5) == B.EDTYPE
    assert f(rows=-1) == f(cols=-1) == f(cols=0) == B.EINVAL
    assert f(rows=0, dz=None, q=None, scale=None, rstd=None, ds=None, dx=None) == B.OK
    assert f(dz=None) == f(q=None) == f(scale=None) == f(rstd=None) == f(dx=None) == B.EINVAL
    assert f(dz=at(0) + 1) == f(ds=at(4) + 1) == f(dx=at(5) + 1) == f(scale=at(2) + 1) == B.EINVAL
    assert f(dt_dz=5) == f(dt=B.FP32, dt_dz=B.BF16) == B.EDTYPE
    assert f(dt_dz=B.FP32, dz=at(0) + 2) == B.EINVAL
    assert f(dt_dz=B.FP32, dx=at(0)) == B.EOVERLAP          # in place only where the types are the same
    assert f(dx=at(0) + 2) == f(dx=at(4) + 2) == f(dx=at(1)) == f(dx=at(2)) == f(dx=at(3)) == B.EOVERLAP


def test_linear_q8_fwd(L):
    def f(dt=B.BF16, m=4, n=32, k=64, q=at(0), scale=at(1), w=at(2), w_scale=at(3), bias=at(4), y=at(5), work=None, size=0):
        return L.linear_q8_fwd(dt, m, n, k, q, scale, w, w_scale, bias, y, work, size, None)
    assert L.lmbp_linear_q8_fwd_bytes(4, 32, 64) == L.lmbp_linear_q8_fwd_bytes(0, 32, 65) == 0   # whole vectors; nothing
    need = L.lmbp_linear_q8_fwd_bytes(4096, 4096, 1023)
    assert need == 8192 * 1024
    odd = dict(m=4096, n=4096, k=1023, work=at(6), size=need)
    assert f(**{**odd, "work": None}) == f(**{**odd, "size": need - 1}) == f(**{**odd, "work": at(6) + 8}) == B.EINVAL
    assert f(**{**odd, "work": at(5)}) == f(**{**odd, "work": at(2)}) == f(**{**odd, "work": at(4)}) == B.EOVERLAP
    assert f(dt=5) == B.EDTYPE
    assert f(m=-1) == f(n=-1) == f(k=-1) == f(m=1 << 31) == f(n=1 << 31) == B.EINVAL
    assert f(k=131072) == B.EINVAL                       # 128 * 128 * 131072 = 2^31
    assert f(m=0, q=None, scale=None, y=None) == f(n=0, w=None, w_scale=None, y=None) == B.OK
    assert f(q=None) == f(scale=None) == f(w=None) == f(w_scale=None) == f(y=None) == B.EINVAL
    assert f(scale=at(1) + 1) == f(w_scale=at(3) + 2) == f(bias=at(4) + 1) == f(y=at(5) + 1) == B.EINVAL
    assert f(y=at(0)) == f(y=at(1)) == f(y=at(2) + 2) == f(y=at(3)) == f(y=at(4)) == B.EOVERLAP


def test_linear_q8_bwd(L):
    need = L.lmbp_linear_q8_bwd_bytes(4, 32, 64)
    assert need >= 4 * 32 + 4 * 4
    assert [L.lmbp_linear_q8_bwd_bytes(*s) for s in ((0, 32, 64), (4, 32, 0), (-1, 2, 3), (4, 131072, 64))] == [0] * 4

    def f(dt=B.BF16, m=4, n=32, k=64, dy=at(0), w=at(1), w_scale=at(2), dx=at(3), work=at(4), size=need, add=None, dt_dx=B.BF16):
        return L.linear_q8_bwd(dt, dt_dx, m, n, k, dy, w, w_scale, add, dx, work, size, None)
    assert f(dt=5) == f(dt_dx=5) == B.EDTYPE
    assert f(add=at(5) + 1) == f(dt_dx=B.FP32, dx=at(3) + 2) == f(dt_dx=B.FP32, add=at(5) + 2) == B.EINVAL
    assert f(add=at(3) + 2) == f(add=at(4)) == B.EOVERLAP
    assert f(m=-1) == f(n=-1) == f(k=-1) == f(m=1 << 31) == f(n=131072) == B.EINVAL
    assert f(m=0, dy=None, dx=None, work=None, size=0) == f(k=0, w=None, dx=None, work=None, size=0) == B.OK
    assert f(dy=None) == f(w=None) == f(w_scale=None) == f(dx=None) == B.EINVAL
    assert f(work=None) == f(size=need - 1) == f(size=-1) == f(work=at(4) + 8) == B.EINVAL
    assert f(dy=at(0) + 1) == f(w_scale=at(2) + 1) == f(dx=at(3) + 1) == B.EINVAL
    assert f(dx=at(0)) == f(dx=at(1)) == f(dx=at(2)) == f(dx=at(4)) == f(work=at(0)) == f(work=at(1)) == B.EOVERLAP


def test_linear_bias_grad(L):
    assert [L.lmbp_linear_bias_grad_bytes(*s) for s in ((0, 8), (8, 0), (-1, 8), (1, 1 << 31), (4, 8))] == [0] * 5
    need = L.lmbp_linear_bias_grad_bytes(1 << 17, 8)
    assert need > 0

    def f(dt=B.BF16, dt_db=B.BF16, m=4, n=32, dy=at(0), db=at(1), work=None, size=0):
        return L.linear_bias_grad(dt, dt_db, m, n, dy, db, work, size, None)
    assert f(dt=5) == f(dt_db=5) == B.EDTYPE
    assert f(m=-1) == f(n=-1) == f(n=1 << 31) == f(m=1 << 60, n=1 << 20) == B.EINVAL
    assert f(n=0, dy=None, db=None) == B.OK
    assert f(dy=None) == f(db=None) == f(dy=at(0) + 1) == f(dt_db=B.FP32, db=at(1) + 2) == B.EINVAL
    big = dict(m=1 << 17, n=8, db=at(0) - 64)
    assert f(**big) == f(**big, work=at(0) - 4096, size=need - 1) == f(**big, work=at(0) - 4088, size=need) == B.EINVAL
    assert f(**big, work=at(0), size=need) == f(db=at(0)) == B.EOVERLAP


def test_the_binding_refuses_what_is_not_on_a_gpu():
    x, q, one = torch.zeros(2, 16), torch.zeros(2, 16, dtype=torch.int8), torch.ones(2)
    for call in (lambda: lmbp.q8_rows(x), lambda: lmbp.q8_values(q, one), lambda: lmbp.msrms_q8_fwd(x, 1e-5),
                 lambda: lmbp.msrms_q8_bwd(x, q, one, one), lambda: lmbp.linear_q8_fwd(q, one, q, one),
                 lambda: lmbp.linear_q8_bwd(x, q, one), lambda: lmbp.linear_bias_grad(x)):
        with pytest.raises(ValueError, match="GPU tensor"):
            call()


def test_modules_refuse_what_is_no_8_bit_layer():
    w, s = torch.zeros(4, 6, dtype=torch.int8), torch.ones(4)
    for bad in ((w.float(), s, None), (w[0], s, None), (w, s.bfloat16(), None), (w, torch.ones(6), None),
                (w, s, torch.zeros(6))):
        with pytest.raises(ValueError):
            lnn.LinearQ8(*bad)
    for bad in ([], [torch.nn.Linear(6, 4)]):
        with pytest.raises(TypeError):
            lnn.MSRMSNormLinearQ8(bad)


def test_module_buffers_and_types():
    layer = lnn.LinearQ8(torch.ones(4, 6, dtype=torch.int8), torch.full((4,), 1.0 + 2.0 ** -20), torch.zeros(4))
    layer.to(torch.bfloat16)
    assert layer.weight.dtype == torch.int8 and layer.bias.dtype == torch.bfloat16
    assert layer.scale.dtype == torch.float32 and (layer.scale == 1.0 + 2.0 ** -20).all()   # not rounded on the way
    assert sorted(layer.state_dict()) == ["bias", "scale", "weight"]
    assert not layer.bias.requires_grad and (layer.in_features, layer.out_features) == (6, 4)
