"""Rotation of part of a head's columns beside columns that are not finite, positions of any size, rows of no sequence and
heads that lie inside each other's rows."""

import math

import pytest
import torch

import paper_2406_16282_amd as lmbp
import plain_heads as P
from paper_2406_16282_amd import binding as B
from paper_2406_16282_amd import nn as lnn
from test_gpu_attention import normal, starts_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5
INF, NAN = math.inf, math.nan


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


# (dim, pairs, interleaved): pieces of 16 and of 8 bytes, element by element, a lane whose pairs turn in part, no pair at all
PART = [(128, 32, False), (64, 16, True), (72, 18, False), (80, 4, True), (96, 21, True), (7, 3, False), (7, 2, True), (40, 5, False), (64, 0, False)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,pairs,interleaved", PART)
def test_columns_that_do_not_turn_are_left_as_they_are(dim, pairs, interleaved, dtype):
    """To the bit: infinities, NaN beside numbers, zeros of either sign."""
    r = B.Rotation([0.7 ** p for p in range(pairs)], None, interleaved)
    x = normal((9, 5, dim), 1).to(dtype)
    clean = x.clone()
    still = range(2 * pairs, dim)
    for i, c in enumerate(still):
        if i % 2 == 0:
            x[i % 9, :, c] = (INF, -INF, NAN)[i // 2 % 3]
        x[(i + 4) % 9, :, c] = -0.0
    pos = torch.arange(9, device=DEV) * 37
    for op in (lmbp.rope_fwd, lmbp.rope_bwd):
        y = op(x, x[:, :2], pos, r)
        want = op(clean, None, pos, r)[0]
        assert torch.equal(bits(y[0][..., 2 * pairs:]), bits(x[..., 2 * pairs:])) and torch.equal(y[0][..., :2 * pairs], want[..., :2 * pairs])
        assert torch.equal(bits(y[1]), bits(y[0][:, :2]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,pairs,interleaved", PART)
def test_norm_beside_columns_that_do_not_turn(dim, pairs, interleaved, dtype):
    """An infinite mean square has rstd 0, which leaves 0 of every finite column and NaN of the infinite one alone; an infinite gradient of a
    column that does not turn reaches the gain of that column alone."""
    if 2 * pairs == dim:
        pytest.skip("every column turns")
    r = B.Rotation([0.7 ** p for p in range(pairs)], None, interleaved)
    x, dy = normal((9, 5, dim), 1).to(dtype), normal((9, 5, dim), 2).to(dtype)
    col = dim - 1
    pos = torch.arange(9, device=DEV) * 37
    one = torch.ones(dim, device=DEV)
    spoilt = x.clone()
    spoilt[4, 2, col] = INF
    for gain in (None, one):
        y, _, rstd, _ = lmbp.msrms_rope_fwd(spoilt, None, EPS, pos, r, gain)
        assert y[4, 2, col].isnan() and (y[4, 2, :col] == 0).all() and rstd[4, 2] == 0
    dy[4, 2, col] = INF
    rstd = lmbp.msrms_rope_fwd(x, None, EPS, pos, r, one)[2]
    dgain = lmbp.msrms_rope_bwd(dy, None, x, None, rstd, None, pos, r, one)[2]
    assert dgain[:col].isfinite().all() and dgain[col].isinf()


@pytest.mark.parametrize("bad", [NAN, INF])
def test_rows_of_no_sequence_may_hold_anything(bad):
    """Padding behind the last start: zeros of output and gradient, the sequences' as without it."""
    heads, kv_heads, dim, lengths = 6, 2, 64, [20, 100, 1, 29]
    n, rows = sum(lengths), sum(lengths) + 11
    r, pos = B.Rotation.of_base(dim), torch.arange(rows, device=DEV)
    qkv, do = normal((rows, heads + 2 * kv_heads, dim), 1), normal((rows, heads, dim), 2)
    qkv[n:], do[n:] = bad, bad
    for eps in (None, EPS):
        m = lnn.QKVAttention(heads, kv_heads, dim, r, eps=eps)
        got = []
        for x in (qkv, qkv[:n].contiguous()):
            x = x.detach().requires_grad_()
            o = m(x, pos[:len(x)], starts_of(lengths))
            got.append((o, *torch.autograd.grad(o, x, do[:len(x)])))
        for a, b in zip(*got):
            assert torch.equal(a[:n], b) and (a[n:] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gain", [False, True])
@pytest.mark.parametrize("dim", [128, 72, 7])
def test_heads_that_get_no_gradient_give_none(dim, gain, dtype):
    """A head that is not finite, whose gradient is 0: zeros, and nothing to the gain's gradient. One that gets a gradient gives NaN."""
    r = B.Rotation([0.7 ** p for p in range(dim // 4)])
    x, dy = normal((9, 5, dim), 1).to(dtype), normal((9, 5, dim), 2).to(dtype)
    pos = torch.arange(9, device=DEV)
    w = (torch.ones(dim, device=DEV),) if gain else ()
    dy[4, 2] = 0.0
    dy[5, 1] = -0.0

    def back(x):
        y, _, rstd, _ = lmbp.msrms_rope_fwd(x, None, EPS, pos, r, *w)
        return lmbp.msrms_rope_bwd(dy, None, x if gain else y, None, rstd, None, pos, r, *w)

    want = back(x)
    x[4, 2, 1], x[5, 1] = INF, NAN
    got = back(x)
    assert torch.equal(got[0], want[0]) and (got[0][4, 2] == 0).all()
    if gain:
        assert torch.equal(got[2], want[2])
    x[6, 3, 0] = NAN
    got = back(x)
    assert got[0][6, 3].isnan().all() and (not gain or got[2].isnan().all())


def test_heads_side_by_side_with_their_keys_and_values():
    """Queries, keys and values of each head side by side ([rows, heads, 3, dim]): turned in place, gradients into one tensor."""
    rows, heads, dim = 70, 4, 64
    r, pos = B.Rotation.of_base(dim), torch.arange(rows, device=DEV)
    qkv, do = normal((rows, heads, 3, dim), 1), normal((rows, heads, dim), 2)
    q, k, v = (t.contiguous() for t in qkv.unbind(2))
    yq, yk = lmbp.rope_fwd(q, k, pos, r)
    x = qkv.clone()
    lmbp.rope_fwd(x[:, :, 0], x[:, :, 1], pos, r, q_out=x[:, :, 0], k_out=x[:, :, 1])
    assert torch.equal(x[:, :, 0], yq) and torch.equal(x[:, :, 1], yk) and torch.equal(x[:, :, 2], v)
    o, lse = lmbp.attention_fwd(yq, yk, v, causal=True)
    want = lmbp.attention_bwd(do, yq, yk, v, o, lse, causal=True)
    for at in (slice(None), slice(0, 1)):   # one row, too
        if at.stop == 1:
            yq, yk, v, o, lse, do, x = yq[:1], yk[:1], v[:1], o[:1], lse[:1], do[:1], x[:1]
            want = lmbp.attention_bwd(do, yq, yk, v, o, lse, causal=True)
        d = torch.full_like(x, 7.0)
        lmbp.attention_bwd(do, x[:, :, 0], x[:, :, 1], x[:, :, 2], o, lse, causal=True, dq=d[:, :, 0], dk=d[:, :, 1], dv=d[:, :, 2])
        assert all(torch.equal(a, b) for a, b in zip(d.unbind(2), want))


TWO_PI = 6283185307179586476925286766559005768394338798750211641949889184615632812572417997256069650684234135964296173026564613294187689219101164463450718816256   # 2 pi 10^150


def exact_angle(pos, freq):
    """pos freq modulo a turn in whole numbers, in radians from -pi to pi."""
    n, d = freq.as_integer_ratio()
    turn = TWO_PI * d
    rest = pos * n * 10 ** 150 % turn
    return (rest - turn if 2 * rest > turn else rest) / turn * 2 * math.pi


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("interleaved", [False, True])
def test_angles_of_positions_of_any_size(dtype, interleaved):
    """Against angles in whole numbers: a frequency is cut to within 1.5 of 2^-64 turns, which a position multiplies, and nothing else is lost."""
    freqs = [1.0, -1.0, 0.3, 1e-4, 10000.0 ** (-5 / 64), 3.0, 1e3, 2.0 ** 40 + 1.0, 2.0 ** 51 + 0.5, 1e-12, 1.0 / 3.0, -2.0 ** -30, 0.0]
    r = B.Rotation(freqs, None, interleaved)
    pos = [0, 1, -1, 12345, 2 ** 24 + 1, -(2 ** 30) - 1, 2 ** 31 - 1, -2 ** 31]
    if dtype == torch.int64:
        pos += [2 ** 40 - 1, 2 ** 50 + 3, -2 ** 53 - 1]
    x = torch.randn(len(pos), 3, 2 * len(freqs), device=DEV)
    t = torch.tensor([[exact_angle(p, f) for f in freqs] for p in pos], dtype=torch.float64, device=DEV)[:, None]
    slack = torch.tensor([abs(p) * 1.5 * 2.0 ** -64 * 2 * math.pi for p in pos], dtype=torch.float64, device=DEV)[:, None, None]
    for op, sign in ((lmbp.rope_fwd, 1), (lmbp.rope_bwd, -1)):
        y, _ = op(x, None, torch.tensor(pos, device=DEV, dtype=dtype), r)
        want = P.turn(x.double(), sign * t, interleaved)
        # 6 u of a pair's size as in any turn; the cut; the 64-bit angle, cosine and sine of the reference (below 2^-48)
        room = (6 * P.U + slack + 2.0 ** -48) * P.pair_size(x.double(), len(freqs), interleaved)
        P.inside(y, want, room + P.U * want.abs(), op.__name__)
