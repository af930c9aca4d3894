"""Attention where keys are not in use, where scores or factors are infinite, and where a group is very large: what the
definition gives, in whichever form the sizes take."""

import math

import pytest
import torch

import paper_2406_16282_amd as lmbp
import plain_heads as P
from test_gpu_attention import check_all, normal, starts_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF, NAN = math.inf, math.nan


# (heads, kv_heads, rows, cache rows, keys in use): a key tile's rows in one share, in several, and a tile that no key in use is in
UNUSED = [(64, 64, 40, 100, 70), (16, 1, 600, 130, 33), (2, 2, 33, 300, 1), (12, 4, 197, 197, 196)]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("what", ["low scores", "infinite do", "NaN q"])
@pytest.mark.parametrize("heads,kv_heads,rows,room,used", UNUSED)
def test_gradients_of_keys_not_in_use_are_zeros(heads, kv_heads, rows, room, used, what, dim, causal):
    """Whatever the queries hold: logarithms of sums far below 0 (a key of zeros would weigh 2^130 and more), rows that are not finite."""
    q, do = normal((2, rows, heads, dim), 1), normal((2, rows, heads, dim), 2)
    k, v = normal((2, room, kv_heads, dim), 3), normal((2, room, kv_heads, dim), 4)
    if what == "low scores":   # every score at most -200 sqrt(dim)
        q, k = q.abs() + 2, -(k.abs() + 100)
    elif what == "infinite do":
        do[:, rows // 2, :, 1] = INF
    else:
        q[:, rows // 3] = NAN
    lens = torch.tensor([used, room], device=DEV, dtype=torch.int32)
    kw = dict(causal=causal, k_lens=lens)
    o, lse = lmbp.attention_fwd(q, k, v, **kw)
    _, dk, dv = lmbp.attention_bwd(do, q, k, v, o, lse, **kw)
    assert (dk[0, used:] == 0).all() and (dv[0, used:] == 0).all()
    if what == "low scores":
        assert lse.max() < -100 and dk.isfinite().all() and dv.isfinite().all()
    # a call that leaves them alone has the same gradients of the keys in use
    mine = [torch.full_like(t, 7.0) for t in (q, k, v)]
    lmbp.attention_bwd(do, q, k, v, o, lse, **kw, dq=mine[0], dk=mine[1], dv=mine[2])
    for got, want in zip(mine[1:], (dk, dv)):
        assert torch.equal(got[0, :used].view(torch.int16), want[0, :used].view(torch.int16)) and (got[0, used:] == 7).all()


def test_a_group_of_many_millions_of_heads():
    """Rows of a key tile behind the last key, times the heads of a group, pass 32 bits: the mask of the keys in use holds. Two queries of 17
    million heads on one key head: the first query's gradient comes to the first key alone."""
    heads = 17_000_000
    room = lambda fill: torch.full((heads, 2, 8), fill, device=DEV, dtype=torch.bfloat16).transpose(0, 1)
    q, o, dq, do = room(0.0), room(7.0), room(7.0), room(0.0)
    do[0] = 1.0
    k = torch.ones(2, 1, 8, device=DEV, dtype=torch.bfloat16)
    v = torch.tensor([1.0, 3.0], device=DEV, dtype=torch.bfloat16)[:, None, None].repeat(1, 1, 8)
    lse = torch.empty(2, heads, device=DEV)
    lmbp.attention_fwd(q, k, v, causal=True, o=o, lse=lse)
    assert (o[0] == 1).all() and (o[1] == 2).all()
    dk, dv = torch.empty_like(k), torch.empty_like(k)
    lmbp.attention_bwd(do, q, k, v, o, lse, causal=True, dq=dq, dk=dk, dv=dv)
    assert (dq == 0).all() and (dk == 0).all() and (dv[1] == 0).all()
    # P is within 4 u of 1; sums of ones are whole numbers: at most 2^24 of them exact, beyond that u each of 512 shares
    assert ((dv[0].double() - heads).abs() <= heads * (P.half(torch.bfloat16) + 520 * P.U)).all()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim,n", [(2, 2, 64, 150), (2, 2, 128, 160), (4, 1, 128, 33), (3, 1, 64, 65), (1, 1, 128, 5), (6, 2, 40, 300)])
def test_a_key_that_weighs_nothing(heads, kv_heads, dim, n, causal):
    """A key that holds an infinity and whose scores are all -inf: no weight and gradients of 0, as one far below the others, also where
    the rows end inside a tile (what is behind them is no row). dq has its infinity times 0 in one column."""
    at, col = 2, 5
    q, do = normal((n, heads, dim), 1), normal((n, heads, dim), 2)
    k, v = normal((n, kv_heads, dim), 3), normal((n, kv_heads, dim), 4)
    q[:, :, col] = 1.0
    kw = dict(causal=causal, q_starts=starts_of([n]))
    k[at, :, col] = -1e4   # weighs 0 in fp32 beside any other key of these
    clean = lmbp.attention_fwd(q, k, v, **kw)
    want = lmbp.attention_bwd(do, q, k, v, *clean, **kw)
    assert (want[2][at] == 0).all()
    k[at, :, col] = -INF
    o, lse = lmbp.attention_fwd(q, k, v, **kw)
    assert torch.equal(o, clean[0]) and torch.equal(lse, clean[1])
    dq, dk, dv = lmbp.attention_bwd(do, q, k, v, o, lse, **kw)
    assert torch.equal(dk, want[1]) and torch.equal(dv, want[2])
    rest = [c for c in range(dim) if c != col]
    sees = at if causal else 0   # the first query that sees the key
    assert torch.equal(dq[..., rest], want[0][..., rest]) and dq[sees:, :, col].isnan().all() and dq[:sees].isfinite().all()


# (heads, kv_heads, rows, keys): few queries in one share and in several, 128 rows to a block in one share and in several
FORMS = [(8, 2, 1, 300), (8, 2, 1, 600), (8, 2, 3, 20000), (1, 1, 256, 16384), (2, 2, 200, 200)]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads,rows,keys", FORMS)
def test_rows_all_of_whose_scores_are_minus_infinity(heads, kv_heads, rows, keys, dim):
    """Scores that overflow: the definition has no weights (NaN) and a logarithm of -inf, in any form; no other row changes."""
    q, k, v = normal((rows, heads, dim), 1), normal((keys, kv_heads, dim), 2), normal((keys, kv_heads, dim), 3)
    k[:, :, 0] = -1024.0
    q[:, :, 0] = 0.0
    clean = lmbp.attention_fwd(q, k, v)
    head = heads - 1
    q[rows // 2, head] = 0.0
    q[rows // 2, head, 0] = 2.0 ** 127
    o, lse = lmbp.attention_fwd(q, k, v)
    assert o[rows // 2, head].isnan().all() and lse[rows // 2, head] == -INF
    keep = torch.ones(rows, heads, dtype=torch.bool, device=DEV)
    keep[rows // 2, head] = False
    assert torch.equal(o[keep], clean[0][keep]) and torch.equal(lse[keep], clean[1][keep])
    # one key with a score among the others has all of the weight, and no key at all gives 0
    k[keys // 3, :, 0] = 0.0
    o, lse = lmbp.attention_fwd(q, k, v)
    assert torch.equal(o[rows // 2, head], v[keys // 3, kv_heads - 1]) and lse[rows // 2, head] == 0
    o, lse = lmbp.attention_fwd(q, k, v, k_lens=torch.zeros(1, device=DEV, dtype=torch.int32))
    assert (o == 0).all() and (lse == -INF).all()


@pytest.mark.parametrize("scale", [2.3e38, 1e-44])
def test_the_largest_and_smallest_scale(scale):
    """Scores of 0 stay 0 and equal weights equal."""
    q, k, v = torch.zeros(40, 2, 64, device=DEV, dtype=torch.bfloat16), normal((70, 2, 64), 1), normal((70, 2, 64), 2)
    v[:] = v[:1]
    o, lse = lmbp.attention_fwd(q, k, v, scale=scale)
    # 70 equal values: P = 1, a sum of 70 in fp32, its reciprocal, the result's rounding
    P.inside(o, v[:1].double().expand(40, 2, 64), (80 * P.U + P.half(torch.bfloat16)) * v[:1].double().abs(), "o")
    P.inside(lse, torch.full((40, 2), math.log(70), dtype=torch.float64, device=DEV), 20 * P.U, "lse")


@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("heads,kv_heads,dim,n,m", [(2, 2, 64, 100, 60), (6, 2, 128, 150, 33), (8, 1, 128, 20, 3)])
def test_queries_that_see_no_key_or_some_reach_only_those(heads, kv_heads, dim, n, m, bad):
    """More queries than keys: those in front see none, whatever they hold, and the first that sees one reaches that key's
    gradients and no later one's."""
    q, do = normal((n, heads, dim), 1), normal((n, heads, dim), 2)
    k, v = normal((m, kv_heads, dim), 3), normal((m, kv_heads, dim), 4)
    o, lse = lmbp.attention_fwd(q, k, v, causal=True)
    want = lmbp.attention_bwd(do, q, k, v, o, lse, causal=True)
    first = n - m   # sees key 0
    for t in (q, do):
        t[:first] = bad
    o2, lse2 = lmbp.attention_fwd(q, k, v, causal=True)
    assert torch.equal(o2, o) and torch.equal(lse2, lse)
    got = lmbp.attention_bwd(do, q, k, v, o2, lse2, causal=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and (got[0][:first] == 0).all()
    q[first, :, 1], do[first, :, 1] = bad, bad
    o2, lse2 = lmbp.attention_fwd(q, k, v, causal=True)
    got = lmbp.attention_bwd(do, q, k, v, o2, lse2, causal=True)
    assert torch.equal(got[0][first + 1:], want[0][first + 1:])
    for a, b in zip(got[1:], want[1:]):
        assert torch.equal(a[1:], b[1:]) and not a[0].isfinite().all()
