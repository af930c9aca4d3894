"""Gradient of a linear layer's bias against sums in 64 bits.

Of small whole numbers every order of additions in fp32 is exact, so those sums are compared
exactly after one rounding to the result's type. Of other numbers a column's m - 1 additions are off
by u = 2^-24 of a partial sum each, at most the sum of the magnitudes, and the store by half a step.
"""

import ctypes

import pytest
import torch

import paper_2406_16282_amd as lmbp
from paper_2406_16282_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]
SIZES = [(0, 5), (1, 1), (1, 4096), (3, 7), (63, 64), (257, 1), (100, 48), (1025, 33), (4097, 256), (700, 1001),
         (20011, 48), (5, 11008), (2048, 1024), (100003, 3), (6000, 4096)]


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", SIZES)
def test_whole_numbers(m, n, dtype, out):
    g = torch.Generator(device=DEV).manual_seed(m + n)
    dy = torch.randint(-8, 9, (m, n), generator=g, device=DEV).to(dtype)
    db = lmbp.linear_bias_grad(dy, out)
    assert db.shape == (n,) and db.dtype == out and torch.equal(db, dy.double().sum(0).to(out))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", [(1, 33), (300, 1001), (8192, 768), (50000, 16)])
def test_any_numbers(m, n, dtype):
    g = torch.Generator(device=DEV).manual_seed(m + n)
    dy = torch.randn(m, n, generator=g, device=DEV).to(dtype)
    want, size = dy.double().sum(0), dy.double().abs().sum(0)
    h = torch.finfo(dtype).eps / 2
    room = (m - 1) * U * size
    assert ((lmbp.linear_bias_grad(dy) - want).abs() <= room + h * (want.abs() + room)).all()
    first = lmbp.linear_bias_grad(dy, torch.float32)
    assert all(torch.equal(lmbp.linear_bias_grad(dy, torch.float32), first) for _ in range(3))


@pytest.mark.parametrize("shift", [1, 2, 3])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", [(9, 64), (3000, 64), (2000, 37)])
def test_any_address_and_nothing_beside_the_result(m, n, dtype, shift):
    src = torch.randint(-8, 9, (m, n), device=DEV).to(dtype)
    buf = torch.full((m * n + 8,), 77, dtype=dtype, device=DEV)
    dy = buf[shift:shift + m * n]
    dy.copy_(src.reshape(-1))
    out = torch.full((n + 8,), 77, dtype=dtype, device=DEV)
    db = out[shift:shift + n]
    L, dt = lmbp.lib(), B.BF16 if dtype == torch.bfloat16 else B.FP32
    need = L.lmbp_linear_bias_grad_bytes(m, n)
    work = torch.full((need + 64,), 77, dtype=torch.uint8, device=DEV)
    assert L.linear_bias_grad(dt, dt, m, n, ctypes.c_void_p(dy.data_ptr()), ctypes.c_void_p(db.data_ptr()),
                              ctypes.c_void_p(work.data_ptr()), need, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == B.OK
    assert torch.equal(db, src.double().sum(0).to(dtype))
    assert (out[:shift] == 77).all() and (out[shift + n:] == 77).all() and (work[need:] == 77).all()
    assert (buf[:shift] == 77).all() and (buf[shift + m * n:] == 77).all()


def test_more_than_2_31_values():
    m, n = 2_200_000, 1024
    dy = torch.zeros(m, n, dtype=torch.bfloat16, device=DEV)
    dy[::100_000] = 1.0
    dy[m - 1] = 2.0
    assert (lmbp.linear_bias_grad(dy, torch.float32) == 24.0).all()


def test_numbers_that_are_not_finite_and_other_shapes():
    dy = torch.ones(2, 50, 40, device=DEV)
    dy[1, 3, 5], dy[0, 7, 6] = float("nan"), float("inf")
    db = lmbp.linear_bias_grad(dy)
    assert db[5].isnan() and db[6] == float("inf")
    keep = [i for i in range(40) if i not in (5, 6)]
    assert (db[keep] == 100.0).all()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = lmbp.linear_bias_grad(dy, stream=side)
    side.synchronize()
    assert torch.equal(got[keep], db[keep])
    for bad in (dy.half(), dy.double(), dy.cpu(), dy.transpose(0, 1)):
        with pytest.raises((ValueError, TypeError)):
            lmbp.linear_bias_grad(bad)
    with pytest.raises((ValueError, TypeError)):
        lmbp.linear_bias_grad(dy, torch.float16)
