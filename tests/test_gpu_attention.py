"""GPU parity of attention against 64 bits (plain_heads.py has the definitions and the bounds). The backward is
compared at the o and lse that the forward gave."""

import math

import pytest
import torch

import paper_2406_16282_amd as lmbp
import plain_heads as P
from paper_2406_16282_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
H = P.half(torch.bfloat16)


def normal(shape, seed, std=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * std).bfloat16()


def starts_of(lengths):
    return torch.tensor([0, *lengths], device=DEV).cumsum(0).int()


def check_all(q, k, v, do, o, lse, grads, lengths, keys, causal, scale, k_at=None):
    """Every sequence and head. q, k, v packed [rows, heads, dim]; k_at: first key rows where they are not the sums."""
    heads, kv_heads = q.shape[1], k.shape[1]
    group = heads // kv_heads
    row = at = 0
    for i, (n, m) in enumerate(zip(lengths, keys)):
        a = slice(row, row + n)
        first = at if k_at is None else k_at[i]
        b = slice(first, first + m)
        for h in range(kv_heads):
            kh, vh = k[b, h], v[b, h]
            sums = None
            for g in range(h * group, (h + 1) * group):
                what = f"sequence {i} ({n}, {m}) head {g}"
                P.check_forward(o[a, g], lse[a, g], q[a, g], kh, vh, causal, scale, what)
                if grads is None:
                    continue
                parts = P.back_with_room(*(t.double() for t in (do[a, g], q[a, g], kh, vh, o[a, g], lse[a, g])), causal, scale)
                dq, room = parts[0], parts[3][0]
                P.inside(grads[0][a, g], dq, room + H * dq.abs(), what + ": dq")
                now = [parts[1], parts[2], *parts[3][1:]]
                sums = now if sums is None else [x + y for x, y in zip(sums, now)]
            if sums is not None:
                for got, want, room, name in ((grads[1][b, h], sums[0], sums[2], "dk"), (grads[2][b, h], sums[1], sums[3], "dv")):
                    P.inside(got, want, room * (1 + group * n * P.U) + H * want.abs(), f"sequence {i} key head {h}: {name}")
        row, at = row + n, at + m


def run(heads, kv_heads, dim, lengths, keys, causal, seed=1, scale=None, size=1.0, train=True, dense=False):
    total, total_k = sum(lengths), sum(keys)
    q, k, v = normal((total, heads, dim), seed, size), normal((total_k, kv_heads, dim), seed + 1, size), normal((total_k, kv_heads, dim), seed + 2)
    do = normal((total, heads, dim), seed + 3, 1e-2)
    scale = dim ** -0.5 if scale is None else scale
    kw = dict(causal=causal, scale=scale)
    if dense:
        n = len(lengths)
        shape = lambda t: t.view(n, -1, *t.shape[1:])
        o, lse = lmbp.attention_fwd(shape(q), shape(k), shape(v), **kw)
        grads = lmbp.attention_bwd(shape(do), shape(q), shape(k), shape(v), o, lse, **kw)
        o, lse, grads = o.flatten(0, 1), lse.flatten(0, 1), [t.flatten(0, 1) for t in grads]
    else:
        kw.update(q_starts=starts_of(lengths), k_starts=starts_of(keys))
        o, lse = lmbp.attention_fwd(q, k, v, **kw)
        grads = lmbp.attention_bwd(do, q, k, v, o, lse, **kw)
    assert o.shape == q.shape and lse.shape == q.shape[:-1] and lse.dtype == torch.float32
    check_all(q, k, v, do, o, lse, grads if train else None, lengths, keys, causal, scale)


# (heads, kv_heads, dim, lengths, key lengths): one row, tile edges on both sides, groups that do not divide a tile,
# more queries than keys, lengths of zero
PACKED = [(1, 1, 64, [1], [1]), (2, 2, 128, [1, 1, 1], [1, 2, 65]), (4, 4, 64, [31, 32, 33], [31, 32, 33]),
          (2, 2, 128, [63, 64, 65], [63, 64, 65]), (2, 1, 128, [127, 128, 129], [127, 128, 129]), (6, 2, 64, [43, 1, 100], [43, 1, 100]),
          (5, 1, 128, [26, 77], [26, 77]), (7, 1, 72, [37, 19, 200], [37, 19, 200]), (8, 1, 8, [50, 3], [50, 3]), (3, 3, 16, [70], [70]),
          (4, 2, 96, [200, 5], [200, 5]), (2, 2, 120, [90, 91], [90, 91]), (8, 2, 128, [5, 17], [300, 17]), (2, 2, 64, [100, 3], [1, 400]),
          (4, 4, 128, [0, 10, 0, 3], [5, 10, 0, 0]), (12, 12, 64, [197, 197], [197, 197]), (16, 2, 128, [1, 1, 1], [700, 1, 65]),
          (2, 1, 40, [300], [513]), (40, 40, 128, [3], [3]), (1, 1, 128, [530], [530])]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("case", PACKED, ids=str)
def test_packed(case, causal):
    print(f"[attention] {case} {causal}", flush=True)
    run(*case, causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim,n,m,count", [(12, 12, 64, 197, 197, 3), (4, 1, 128, 65, 200, 2), (2, 2, 128, 1, 1000, 2),
                                                          (3, 3, 56, 40, 7, 4), (1, 1, 128, 1100, 1100, 1)])
def test_dense(heads, kv_heads, dim, n, m, count, causal):
    run(heads, kv_heads, dim, [n] * count, [m] * count, causal, dense=True)


@pytest.mark.parametrize("size,scale", [(8.0, None), (1e-3, None), (1.0, 3.0), (1.0, 1e-4), (30.0, 1.0)])
def test_large_and_small_scores(size, scale):
    """Rows whose softmax is one key, and rows that are nearly even."""
    run(4, 2, 64, [150], [150], True, size=size, scale=scale)
    run(4, 2, 128, [1], [900], False, size=size, scale=scale)


@pytest.mark.parametrize("heads,kv_heads,dim,n", [(8, 8, 128, 1), (8, 1, 64, 1), (8, 2, 128, 3), (32, 2, 128, 4), (12, 4, 96, 16)])
@pytest.mark.parametrize("keys", [[1, 4000, 65], [20000], [0, 64, 5000, 129]])
def test_few_queries_behind_many_keys(heads, kv_heads, dim, n, keys):
    keys = [m + n if m else 0 for m in keys]
    run(heads, kv_heads, dim, [n] * len(keys), keys, True, train=False)
    run(heads, kv_heads, dim, [n] * len(keys), keys, False, train=False)


@pytest.mark.parametrize("n", [1, 5])
def test_padded_cache(n):
    """Sequences at the front of a cache's rows; what lies behind them is not read."""
    lens = [7, 400, 64, 1, 0, 129]
    room, heads, kv_heads, dim = 410, 8, 2, 128
    q = normal((len(lens), n, heads, dim), 1)
    k, v = normal((len(lens), room, kv_heads, dim), 2), normal((len(lens), room, kv_heads, dim), 3)
    for i, m in enumerate(lens):
        k[i, m:], v[i, m:] = float("nan"), float("inf")
    used = torch.tensor(lens, dtype=torch.int32, device=DEV)
    for causal in (True, False):
        o, lse = lmbp.attention_fwd(q, k, v, causal=causal, k_lens=used)
        check_all(q.flatten(0, 1), k.flatten(0, 1), v.flatten(0, 1), None, o.flatten(0, 1), lse.flatten(0, 1), None, [n] * len(lens), lens,
                  causal, dim ** -0.5, [i * room for i in range(len(lens))])
        do = normal(q.shape, 4)
        grads = lmbp.attention_bwd(do, q, k, v, o, lse, causal=causal, k_lens=used)
        check_all(q.flatten(0, 1), k.flatten(0, 1), v.flatten(0, 1), do.flatten(0, 1), o.flatten(0, 1), lse.flatten(0, 1),
                  [t.flatten(0, 1) for t in grads], [n] * len(lens), lens, causal, dim ** -0.5, [i * room for i in range(len(lens))])
        for i, m in enumerate(lens):
            assert (grads[1][i, m:] == 0).all() and (grads[2][i, m:] == 0).all()
    # lengths beyond the cache, and below nothing: as much as there is
    wrong = torch.tensor([10 ** 9, -5, 64, 1, 0, 129], dtype=torch.int32, device=DEV)
    k, v = normal(k.shape, 2), normal(v.shape, 3)
    o, lse = lmbp.attention_fwd(q, k, v, k_lens=wrong)
    assert o.isfinite().all() and (o[1] == 0).all() and (lse[1] == -math.inf).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dim", [64, 128])
def test_what_a_query_does_not_see_may_hold_anything(dim, bad):
    """Causal: an infinity or NaN of a later token, within the tile of the query, reaches no earlier one."""
    n, at, heads = 150, 77, 2
    q, k, v, do = (normal((n, heads, dim), i) for i in range(4))
    starts = starts_of([n])
    kw = dict(causal=True, q_starts=starts)
    clean = lmbp.attention_fwd(q, k, v, **kw)
    grads = lmbp.attention_bwd(do, q, k, v, *clean, **kw)
    for spoil in ("k", "v", "both"):
        k2, v2 = k.clone(), v.clone()
        if spoil != "v":
            k2[at, :, 3] = bad
        if spoil != "k":
            v2[at, :, 5] = bad
            v2[at, 0, 6] = bad
        o, lse = lmbp.attention_fwd(q, k2, v2, **kw)
        assert torch.equal(o[:at], clean[0][:at]) and torch.equal(lse[:at], clean[1][:at])
        want, ref, _, _ = P.attend(q[:, 0].double(), k2[:, 0].double(), v2[:, 0].double(), True, dim ** -0.5)
        if spoil == "v":   # the values that see it, and only those
            assert torch.equal(o[:, 0].isfinite(), want.isfinite())
            assert torch.equal(o[at:, 0, 5].isnan(), want[at:, 5].isnan()) and torch.equal(lse, clean[1])
        # gradients of the tokens in front: as if the sequence ended there, where nothing behind sees them either
        d2 = do.clone()
        d2[at:] = 0
        q2 = q.clone()
        q2[at:] = bad
        got = lmbp.attention_bwd(d2[:at].contiguous(), q[:at].contiguous(), k2[:at].contiguous(), v2[:at].contiguous(), o[:at].contiguous(),
                                 lse[:at].contiguous(), causal=True, q_starts=starts_of([at]))
        dq = lmbp.attention_bwd(do, q, k2, v2, o, lse, **kw)[0]
        assert torch.equal(dq[:at], grads[0][:at])
        assert all(t.isfinite().all() for t in got)
    # queries that a key is not seen by: a row in front, spoilt, reaches no later key's gradients
    q2, do2 = q.clone(), do.clone()
    q2[at, :, 3], do2[at, :, 2] = bad, bad
    o, lse = lmbp.attention_fwd(q2, k, v, **kw)
    _, dk, dv = lmbp.attention_bwd(do2, q2, k, v, o, lse, **kw)
    assert torch.equal(dk[at + 1:], grads[1][at + 1:]) and torch.equal(dv[at + 1:], grads[2][at + 1:])
    assert not dk[at].isfinite().all()
    keep = [t for t in range(n) if t != at]
    assert torch.equal(o[keep], clean[0][keep])


def test_spoilt_rows_of_another_sequence():
    lengths = [70, 50, 64]
    q, k, v, do = (normal((sum(lengths), 2, 64), i) for i in range(4))
    kw = dict(causal=False, q_starts=starts_of(lengths))
    clean = lmbp.attention_fwd(q, k, v, **kw)
    want = lmbp.attention_bwd(do, q, k, v, *clean, **kw)
    for t in (q, k, v, do):
        t[70:120] = float("nan")
    o, lse = lmbp.attention_fwd(q, k, v, **kw)
    got = lmbp.attention_bwd(do, q, k, v, o, lse, **kw)
    rest = [*range(70), *range(120, 184)]
    assert torch.equal(o[rest], clean[0][rest]) and all(torch.equal(a[rest], b[rest]) for a, b in zip(got, want))


@pytest.mark.parametrize("group", [1, 3])
def test_rows_of_no_sequence(group):
    """Rows behind the last sequence: zeros in results that are allocated, left alone in those that are given."""
    lengths, rows = [30, 100], 200
    heads, kv_heads, dim = 2 * group, 2, 64
    q, do = normal((rows, heads, dim), 1), normal((rows, heads, dim), 2)
    k, v = normal((rows, kv_heads, dim), 3), normal((rows, kv_heads, dim), 4)
    kw = dict(causal=True, q_starts=starts_of(lengths))
    o, lse = lmbp.attention_fwd(q, k, v, **kw)
    assert (o[130:] == 0).all() and (lse[130:] == -math.inf).all()
    grads = lmbp.attention_bwd(do, q, k, v, o, lse, **kw)
    assert all((t[130:] == 0).all() for t in grads)
    check_all(q, k, v, do, o, lse, grads, lengths, lengths, True, dim ** -0.5)
    mine, mine_lse = torch.full_like(o, 7.0), torch.full_like(lse, 7.0)
    lmbp.attention_fwd(q, k, v, **kw, o=mine, lse=mine_lse)
    assert torch.equal(mine[:130], o[:130]) and (mine[130:] == 7).all() and (mine_lse[130:] == 7).all()
    given = [torch.full_like(t, 7.0) for t in (q, k, v)]
    lmbp.attention_bwd(do, q, k, v, o, lse, **kw, dq=given[0], dk=given[1], dv=given[2])
    assert all(torch.equal(a[:130], b[:130]) and (a[130:] == 7).all() for a, b in zip(given, grads))


@pytest.mark.parametrize("starts", [[0, 50, 20, 90], [0, -3, 40, 10 ** 9], [5, 60, 60, 90], [90, 0, 0, 0]])
def test_starts_that_are_wrong_stay_inside(starts):
    q, k, v = (normal((90, 2, 64), i) for i in range(3))
    s = torch.tensor(starts, dtype=torch.int32, device=DEV)
    guard = torch.full((90 * 2 * 64 + 2048,), 7.0, device=DEV, dtype=torch.bfloat16)
    o = guard[1024:-1024].view(90, 2, 64)
    lse = torch.zeros(90, 2, device=DEV)
    lmbp.attention_fwd(q, k, v, causal=True, q_starts=s, o=o, lse=lse)
    torch.cuda.synchronize()
    assert (guard[:1024] == 7).all() and (guard[-1024:] == 7).all()


def test_strides():
    """Parts of one projection's output, heads in front of rows, gradients into one tensor: the dense results."""
    rows, heads, kv_heads, dim = 100, 6, 2, 64
    qkv = normal((rows, heads + 2 * kv_heads, dim), 1)
    q, k, v = qkv.split((heads, kv_heads, kv_heads), 1)
    do = normal((rows, heads, dim), 2)
    kw = dict(causal=True)
    o, lse = lmbp.attention_fwd(q.contiguous(), k.contiguous(), v.contiguous(), **kw)
    want = lmbp.attention_bwd(do, q.contiguous(), k.contiguous(), v.contiguous(), o, lse, **kw)
    got = lmbp.attention_fwd(q, k, v, **kw)
    assert torch.equal(got[0], o) and torch.equal(got[1], lse)
    d = torch.full_like(qkv, 7.0)
    dq, dk, dv = d.split((heads, kv_heads, kv_heads), 1)
    lmbp.attention_bwd(do, q, k, v, o, lse, **kw, dq=dq, dk=dk, dv=dv)
    assert all(torch.equal(a, b) for a, b in zip((dq, dk, dv), want))
    first = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.zeros(heads, rows, dim, device=DEV, dtype=torch.bfloat16).transpose(0, 1)
    got = lmbp.attention_fwd(first(q), first(k), first(v), **kw, o=out, lse=torch.empty_like(lse))
    assert torch.equal(got[0], o)
    got = lmbp.attention_bwd(first(do), first(q), first(k), first(v), first(o), lse, **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # one key head for all, read through a stride of 0
    one = lmbp.attention_fwd(q, k[:, :1].expand(rows, 2, dim), v[:, :1].expand(rows, 2, dim), **kw)
    copies = [t[:, :1].expand(rows, 2, dim).contiguous() for t in (k, v)]
    assert torch.equal(one[0], lmbp.attention_fwd(q, *copies, **kw)[0])


def test_gradients_of_shared_heads_are_split_over_rows():
    """One key head for many queries: the sums of dk and dv are formed in shares."""
    plan = B._Attention(1, 16, 1, 64, 600, 130, None, None, None, 0.125, 1, 0)
    import ctypes
    alone = B._Attention(64, 16, 16, 64, 64 * 600, 64 * 130, None, None, None, 0.125, 1, 0)
    size = lmbp.lib().lmbp_attention_bwd_bytes
    assert size(ctypes.byref(plan)) > 600 * 16 * 8 + 100 and size(ctypes.byref(alone)) == 64 * 600 * 16 * 8
    run(16, 1, 64, [600], [130], False)
    run(16, 1, 128, [600, 40], [600, 40], True)
    run(24, 2, 72, [700], [64], True)


def test_same_results_every_time():
    lengths = [300, 5, 700]
    q, do = normal((1005, 8, 128), 1), normal((1005, 8, 128), 2)
    k, v = normal((1005, 1, 128), 3), normal((1005, 1, 128), 4)
    kw = dict(causal=True, q_starts=starts_of(lengths))
    o, lse = lmbp.attention_fwd(q, k, v, **kw)
    first = lmbp.attention_bwd(do, q, k, v, o, lse, **kw)
    for _ in range(3):
        o2, lse2 = lmbp.attention_fwd(q, k, v, **kw)
        again = lmbp.attention_bwd(do, q, k, v, o, lse, **kw)
        assert torch.equal(o, o2) and torch.equal(lse, lse2) and all(torch.equal(a, b) for a, b in zip(first, again))
    for _ in range(2):   # the keys in shares
        a, b = (lmbp.attention_fwd(q[:1].contiguous(), k, v)[0] for _ in range(2))
        assert torch.equal(a, b)


def test_long_sequence_sampled():
    """5000 tokens: every query's row against 64 bits at a few heads and rows."""
    n = 5000
    q, k, v = normal((n, 2, 128), 1), normal((n, 2, 128), 2), normal((n, 2, 128), 3)
    o, lse = lmbp.attention_fwd(q, k, v, causal=True)
    for rows in (slice(0, 130), slice(2500, 2600), slice(4900, 5000)):
        P.check_forward(o[rows, 1], lse[rows, 1], q[rows, 1], k[:rows.stop, 1], v[:rows.stop, 1], True, 128 ** -0.5, str(rows))


def test_refusals():
    q, k = normal((10, 4, 64), 1), normal((10, 2, 64), 2)
    s = starts_of([4, 6])
    f = lmbp.attention_fwd
    for call in (lambda: f(q, k, k[:9]), lambda: f(q, k[..., :56], k[..., :56]), lambda: f(q, normal((10, 3, 64), 1), normal((10, 3, 64), 1)),
                 lambda: f(q, k, k, q_starts=s.long()), lambda: f(q, k, k, q_starts=s, k_starts=s[:2]),
                 lambda: f(q, k, k, k_lens=s), lambda: f(q, k, k, q_starts=s.cpu()), lambda: f(q[0], k, k),
                 lambda: f(q.view(2, 5, 4, 64), k.view(1, 10, 2, 64), k.view(1, 10, 2, 64)), lambda: f(q, k, k, o=q[:5]),
                 lambda: f(q.transpose(1, 2), k, k), lambda: lmbp.attention_bwd(q[:5], q, k, k, q, torch.zeros(10, 4, device=DEV)),
                 lambda: lmbp.attention_bwd(q, q, k, k, q, torch.zeros(10, 3, device=DEV))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: f(q.float(), k.float(), k.float()), lambda: f(q, k.float(), k), lambda: f(q, k, k, q_starts=[0, 4, 10])):
        with pytest.raises(TypeError):
            call()
    wide, odd = normal((10, 4, 136), 1), normal((10, 4, 12), 1)
    shifted = torch.zeros(10 * 4 * 64 + 1, device=DEV, dtype=torch.bfloat16)[1:].view(10, 4, 64)
    for call in (lambda: f(wide, wide, wide), lambda: f(odd, odd, odd), lambda: f(q, k, k, scale=0.0), lambda: f(q, k, k, scale=-1.0),
                 lambda: f(shifted, k, k), lambda: f(q, k, k, o=q)):
        with pytest.raises(B.LmbpError):
            call()


def test_no_rows():
    q, k = normal((0, 4, 64), 1), normal((5, 4, 64), 2)
    o, lse = lmbp.attention_fwd(q, k, k)
    assert o.shape == (0, 4, 64) and lse.shape == (0, 4)
    dq, dk, dv = lmbp.attention_bwd(q, q, k, k, o, lse)
    assert dq.shape == q.shape and (dk == 0).all() and (dv == 0).all()
    o, lse = lmbp.attention_fwd(k, q, q)
    assert (o == 0).all() and (lse == -math.inf).all()
    dq, dk, dv = lmbp.attention_bwd(k, k, q, q, o, lse)
    assert (dq == 0).all() and dk.shape == q.shape
