"""The 64-bit definitions that the GPU tests compare with: their gradients against differences, on the CPU."""

import math

import pytest
import torch

import plain_heads as P


def differences(f, x, g, step=1e-5):
    """Gradient of sum(f(x) g) by central differences."""
    out = torch.zeros_like(x)
    flat, res = x.reshape(-1), out.reshape(-1)
    for i in range(flat.numel()):
        keep = flat[i].item()
        flat[i] = keep + step
        up = (f() * g).sum()
        flat[i] = keep - step
        down = (f() * g).sum()
        flat[i] = keep
        res[i] = (up - down) / (2 * step)
    return out


@pytest.mark.parametrize("nq,nk,causal", [(3, 3, False), (4, 4, True), (2, 5, True), (5, 2, True), (1, 1, True), (1, 4, False)])
def test_attention_gradients_are_those_of_differences(nq, nk, causal):
    g = torch.Generator().manual_seed(nq * 10 + nk)
    q, k, v, do = (torch.randn(n, 3, generator=g, dtype=torch.float64) for n in (nq, nk, nk, nq))
    scale = 0.7
    o, lse, _, _ = P.attend(q, k, v, causal, scale)
    got = P.attend_back(do, q, k, v, o, lse, causal, scale)[:3]
    for t, d in zip((q, k, v), got):
        want = differences(lambda: P.attend(q, k, v, causal, scale)[0], t, do)
        assert (d - want).abs().max() < 1e-8


def test_attention_rows_that_see_nothing():
    q, k, v = torch.randn(4, 2, dtype=torch.float64), torch.randn(2, 2, dtype=torch.float64), torch.randn(2, 2, dtype=torch.float64)
    o, lse, _, _ = P.attend(q, k, v, True, 1.0)
    assert (o[:2] == 0).all() and (lse[:2] == -math.inf).all() and lse[2:].isfinite().all()
    assert (o[2] == v[0]).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("eps,gain", [(None, False), (1e-3, False), (1e-3, True)])
def test_norm_and_rotation_gradients(interleaved, eps, gain):
    g = torch.Generator().manual_seed(5)
    x, dy = (torch.randn(3, 2, 7, generator=g, dtype=torch.float64) for _ in range(2))
    w = torch.randn(7, generator=g, dtype=torch.float64) if gain else torch.ones(7, dtype=torch.float64)
    t = P.angles(torch.tensor([[0, 5, -3], [7, 1, 2]]), [1.0, 0.3, 0.01], [0, 1, 0], 3)

    def f():
        return P.turn((P.norm(x, eps)[0] if eps else x) * w, t, interleaved)

    back = P.turn(dy, -t, interleaved)
    if eps is None:
        dx = back
    else:
        z, rstd = P.norm(x, eps)
        dx = P.norm_back(back * w, z, rstd)
        if not gain:   # and from the turned output alone
            y = f()
            along = (y * dy).mean(-1, keepdim=True)
            assert (dx - P.turn(rstd * (dy - y * along), -t, interleaved)).abs().max() < 1e-12
        else:
            assert ((back * z).sum((0, 1)) - differences(f, w, dy)).abs().max() < 1e-7
    assert (dx - differences(f, x, dy)).abs().max() < 1e-7
    # the rotation of a pair as a complex number
    i = torch.arange(3)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + 3)
    want = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.ones_like(t), t)
    y = P.turn(x, t, interleaved)
    assert (torch.complex(y[..., a], y[..., b]) - want).abs().max() < 1e-12 and (y[..., 6] == x[..., 6]).all()
