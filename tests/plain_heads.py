"""Rotary positions, norms of heads and attention from their definitions, in 64 bits, with the bounds that the
kernels' roundings are held to. Tensors of heads are [..., heads, dim]; any device.

Bounds. u = 2^-24 (half a step of fp32), h half a step of the result's type. A sum of n products in fp32, in any
order, is within (n + 1) u of the sum of the products' magnitudes (first order; a factor of 1.01 stands for the rest).
Magnitudes below TINY = 2^-126, the smallest normal number of fp32 and bf16, may be taken as 0 wherever a value is formed
(the exponential's result does, so may a factor, a product, a sum or a result): each such value is off by TINY more.
"""

import math

import torch

U = 2.0 ** -24
TINY = 2.0 ** -126


def half(t):
    return torch.finfo(t).eps / 2


def inside(got, want, room, what):
    """Every value within ``room`` of ``want``; where want is not finite, the same there."""
    got = got.double()
    same = (got == want) | (got.isnan() & want.isnan())
    ok = torch.where(want.isfinite(), (got - want).abs() <= 1.01 * room + TINY, same)
    assert ok.all(), (f"{what}: {int((~ok).sum())} of {ok.numel()} values outside, first {(~ok).nonzero()[0].tolist()}: "
                      f"{got[~ok][0].item()!r} for {want[~ok][0].item()!r}")


# ------------------------------------------------------------------------- rotation and norm

def angles(positions, freqs, axes, rows):
    """[rows, 1, pairs]."""
    pairs = len(freqs)
    if pairs == 0:
        return torch.zeros(rows, 1, 0, dtype=torch.float64, device=positions.device if positions is not None else None)
    p = positions.reshape(-1, rows)[torch.tensor(axes if axes is not None else [0] * pairs, device=positions.device)]
    return (p.double() * torch.tensor(freqs, dtype=torch.float64, device=p.device)[:, None]).t()[:, None]


def turn(x, t, interleaved):
    """x [rows, heads, dim] in 64 bits by the angles t."""
    pairs = t.shape[-1]
    i = torch.arange(pairs, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
    y = x.clone()
    y[..., a] = x[..., a] * t.cos() - x[..., b] * t.sin()
    y[..., b] = x[..., a] * t.sin() + x[..., b] * t.cos()
    return y


def pair_size(x, pairs, interleaved):
    """|a| + |b| of every column's pair."""
    i = torch.arange(pairs, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
    size = x.abs().clone()
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return size


def norm(x, eps):
    rstd = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    return x * rstd, rstd


def norm_back(dz, z, rstd):
    return rstd * (dz - z * (z * dz).mean(-1, keepdim=True))


# ---------------------------------------------------------------------------------- attention

def visible(nq, nk, causal, device):
    if not causal:
        return torch.ones(nq, nk, dtype=torch.bool, device=device)
    return torch.arange(nk, device=device)[None] <= torch.arange(nq, device=device)[:, None] + (nk - nq)


def attend(q, k, v, causal, scale):
    """One head of one sequence, [n, dim] in 64 bits: (o, lse, P, S). What a query does not see does not count,
    whatever it holds."""
    see = visible(q.shape[0], k.shape[0], causal, q.device)
    s = torch.where(see, scale * (q @ k.t()), -math.inf)
    lse = torch.logsumexp(s, 1) if k.shape[0] else torch.full((q.shape[0],), -math.inf, dtype=q.dtype, device=q.device)
    p = torch.where(see, torch.exp(s - lse[:, None]), 0.0)
    if v.isfinite().all():
        return p @ v, lse, p, s
    return torch.stack([p[i, see[i]] @ v[see[i]] for i in range(q.shape[0])]), lse, p, s


def attend_back(do, q, k, v, o, lse, causal, scale):
    """(dq, dk, dv, D, P, dS) from the output and lse as they are held."""
    see = visible(q.shape[0], k.shape[0], causal, q.device)
    p = torch.where(see, torch.exp(scale * (q @ k.t()) - lse[:, None]), 0.0)
    d = (do * o).sum(1, keepdim=True)
    ds = torch.where(see, p * (do @ v.t() - d), 0.0)
    return scale * ds @ k, scale * ds.t() @ q, p.t() @ do, d, p, ds


def _exponent_error(q, k, s, lse, scale):
    """Of exp's argument in fp32: the product's sum, the factor scale log2(e) and its product, lse log2(e), the
    difference; and the exponential's own 2 u."""
    size = scale * (q.abs() @ k.abs().t())
    return (q.shape[1] + 2) * U * size + 4 * U * (s.abs() + lse.abs()[:, None]) + 4 * U


def check_forward(o, lse, q, k, v, causal, scale, what):
    """o [nq, dim] and lse [nq] of one head against 64 bits."""
    q, k, v = q.double(), k.double(), v.double()
    want, ref, p, s = attend(q, k, v, causal, scale)
    see = visible(q.shape[0], k.shape[0], causal, q.device)
    s = torch.where(see, s, 0.0)
    base = torch.where(ref.isfinite(), ref, 0.0)
    e = torch.where(see, _exponent_error(q, k, s, base, scale), 0.0)
    n = k.shape[0]
    # sum of P: its terms' errors and the sum's; P as a factor: rounded to bf16, the products' sum
    sums = (p * e).sum(1) + (n + 2) * U
    # (exponentials are relative to a maximum that may be 2^8 behind the largest)
    room = n * TINY + (p * (e + half(torch.bfloat16) + (n + 4) * U) + 2 ** 9 * TINY) @ v.abs() + want.abs() * (sums[:, None] + half(torch.bfloat16))
    inside(o, want, room, what + ": o")
    inside(lse, ref, sums + 4 * U * (base.abs() + 1), what + ": lse")


def check_backward(grads, do, q, k, v, o, lse, causal, scale, what):
    """dq, dk, dv of one head of one sequence (one query head to the key head) from o and lse as the forward gave them."""
    do, q, k, v, o, lse = (t.double() for t in (do, q, k, v, o, lse))
    dq, dk, dv, rooms = back_with_room(do, q, k, v, o, lse, causal, scale)
    h = half(torch.bfloat16)
    for got, want, room, name in zip(grads, (dq, dk, dv), rooms, ("dq", "dk", "dv")):
        inside(got, want, room + h * want.abs(), f"{what}: {name}")


def back_with_room(do, q, k, v, o, lse, causal, scale):
    """dq, dk, dv in 64 bits and the room for their errors before the last rounding (to be added up over the heads
    that share a key head)."""
    dq, dk, dv, d, p, ds = attend_back(do, q, k, v, o, lse, causal, scale)
    see = visible(q.shape[0], k.shape[0], causal, q.device)
    h, dim = half(torch.bfloat16), q.shape[1]
    base = torch.where(lse.isfinite(), lse, 0.0)
    e = torch.where(see, _exponent_error(q, k, torch.where(see, scale * (q @ k.t()), 0.0), base, scale), 0.0)
    diff = (dim + 2) * U * (do.abs() @ v.abs().t() + (do.abs() * o.abs()).sum(1, keepdim=True))
    nq, nk = q.shape[0], k.shape[0]
    ds_room = torch.where(see, ds.abs() * (e + h + 4 * U) + p * diff + TINY * (2 + (do @ v.t() - d).abs()), 0.0)
    rooms = (scale * (ds_room + (nk + 4) * U * ds.abs()) @ k.abs(), scale * (ds_room + (nq + 4) * U * ds.abs()).t() @ q.abs(),
             (p * (e + h + (nq + 6) * U) + 2 * TINY).t() @ do.abs())
    return dq, dk, dv, [r + (n + 2) * TINY * max(1.0, scale) for r, n in zip(rooms, (nk, nq, nq))]
