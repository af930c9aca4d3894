"""Rotary positions, norms of heads and attention where offsets pass 32 bits, with many sequences, from several threads
and behind a growing cache."""

import math
import threading

import pytest
import torch

import paper_2406_16282_amd as lmbp
import plain_heads as P
import test_gpu_rope as rope
from test_gpu_attention import normal, run, starts_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def apart(parts, rows, pitch):
    """Copies of ``parts`` [rows, heads, dim] side by side in rows of ``pitch`` elements, and empty places like them."""
    room = torch.empty(rows * pitch, device=DEV, dtype=parts[0].dtype).view(rows, pitch)
    at, out = 0, []
    for t in (*parts, *parts):
        n = t.shape[1] * t.shape[2]
        out.append(room[:, at:at + n].unflatten(1, t.shape[1:]))
        at += n
    assert at <= pitch and room.data_ptr() % 16 == 0
    for t, place in zip(parts, out):
        place.copy_(t)
    return out[:len(parts)], out[len(parts):]


@pytest.mark.parametrize("starts", [None, [70, 1, 229]])
def test_rows_gibibytes_apart(starts):
    """Layouts do not change results: rows 16 MiB apart, the last beyond 2^32 bytes and 2^31 elements."""
    rows, pitch = 300, (1 << 23) - 8
    q, k, v, do = (normal((rows, h, 128), i) for i, h in enumerate((4, 2, 2, 4)))
    kw = dict(causal=True) if starts is None else dict(causal=True, q_starts=starts_of(starts))
    o, lse = lmbp.attention_fwd(q, k, v, **kw)
    grads = lmbp.attention_bwd(do, q, k, v, o, lse, **kw)
    (fq, fk, fv, fdo, fo), (dq, dk, dv, o2, _) = apart((q, k, v, do, o), rows, pitch)
    assert (fq[-1].data_ptr() - fq[0].data_ptr()) > 1 << 32
    lse2 = torch.empty_like(lse)
    lmbp.attention_fwd(fq, fk, fv, o=o2, lse=lse2, **kw)
    assert torch.equal(o2, o) and torch.equal(lse2, lse)
    lmbp.attention_bwd(fdo, fq, fk, fv, fo, lse, dq=dq, dk=dk, dv=dv, **kw)
    for got, want in zip((dq, dk, dv), grads):
        assert torch.equal(got, want)
    few = lmbp.attention_fwd(q[-1:], k, v)
    got = lmbp.attention_fwd(fq[-1:], fk, fv)
    assert torch.equal(got[0], few[0]) and torch.equal(got[1], few[1])


@pytest.mark.parametrize("dim", [64, 33])
def test_rotation_of_rows_gibibytes_apart(dim):
    rows, pitch = 300, (1 << 23) - 8
    q, k = normal((rows, 3, dim), 1), normal((rows, 1, dim), 2)
    at, turn, gain = torch.arange(rows, device=DEV), lmbp.Rotation.of_base(dim // 2 * 2), normal((dim,), 3)
    (fq, fk), (oq, ok) = apart((q, k), rows, pitch)
    for back in (lmbp.rope_fwd, lmbp.rope_bwd):
        back(fq, fk, at, turn, oq, ok)
        assert all(torch.equal(a, b) for a, b in zip((oq, ok), back(q, k, at, turn)))
    for g in ((), (gain, gain)):
        want = lmbp.msrms_rope_fwd(q, k, 1e-6, at, turn, *g)
        got = lmbp.msrms_rope_fwd(fq, fk, 1e-6, at, turn, *(g or (None, None)), oq, ok)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_cache_of_more_than_32_bits():
    """One token behind 540001 keys of 32 heads: 4.4 GB of each. The first and the last head against 64 bits."""
    keys, heads = 540001, 32
    k, v = (torch.empty(1, keys, heads, 128, device=DEV, dtype=torch.bfloat16).normal_(generator=torch.Generator(DEV).manual_seed(i)) for i in (1, 2))
    q = normal((1, 1, heads, 128), 3)
    used = torch.tensor([keys - 2], device=DEV, dtype=torch.int32)
    o, lse = lmbp.attention_fwd(q, k, v, causal=True, k_lens=used)
    for h in (0, heads - 1):
        P.check_forward(o[0, :, h], lse[0, :, h], q[0, :, h], k[0, :keys - 2, h], v[0, :keys - 2, h], True, 128 ** -0.5, f"head {h}")


@pytest.mark.parametrize("count", [63, 64, 65, 130])
def test_many_sequences(count):
    lengths = [(11 * i * i + 3 * i) % 47 for i in range(count)]
    lengths[5], lengths[count - 2] = 300, 260
    run(2, 1, 64, lengths, lengths, True)


def test_many_sequences_of_other_keys():
    lengths = [(7 * i) % 13 for i in range(62)]
    run(4, 2, 64, lengths, [n + (5 * i) % 90 for i, n in enumerate(lengths)], True)


def test_two_threads():
    work = [[normal((50 + 30 * i, h, 64), 10 * i + h) for h in (8, 2, 2)] for i in range(2)]
    at, turn = torch.arange(80, device=DEV), lmbp.Rotation.of_base(64)

    def step(q, k, v):
        q, k = lmbp.rope_fwd(q, k, at[:q.shape[0]], turn)
        o, lse = lmbp.attention_fwd(q, k, v, True)
        return [q, k, o, lse, *lmbp.attention_bwd(o, q, k, v, o, lse, True), *lmbp.attention_fwd(q[-1:], k, v)]

    want = [step(*w) for w in work]
    torch.cuda.synchronize()
    wrong, errors = [], []

    def body(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(30):
                    got = step(*work[i])
                    wrong.extend(n for n, (a, b) in enumerate(zip(got, want[i])) if not torch.equal(a, b))
        except Exception as e:   # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=body, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    assert not wrong and not errors


def test_a_captured_token_behind_a_growing_cache():
    """One graph takes the tokens one after the other: the position, the number of keys in use and the cache change in place."""
    heads, kv, room, dim = 8, 2, 4000, 128
    cache = normal((2, 2, room, kv, dim), 1)
    new = normal((2, 1, heads + 2 * kv, dim), 2)
    used, at = torch.zeros(2, device=DEV, dtype=torch.int32), torch.zeros(2, device=DEV, dtype=torch.int64)
    turn = lmbp.Rotation.of_base(dim)

    def token():
        q, _, _, _ = lmbp.msrms_rope_fwd(new[:, :, :heads], None, 1e-6, at, turn)
        return lmbp.attention_fwd(q, cache[0], cache[1], True, k_lens=used)

    token()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = token()
    for n in ([1, 3], [700, 65], [4000, 2], [0, 4000]):
        used.copy_(torch.tensor(n)), at.copy_(torch.tensor(n) + 5), new.copy_(normal(new.shape, n[0]))
        graph.replay()
        torch.cuda.synchronize()
        want = token()
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1]), n
        for i in range(2):
            q = lmbp.msrms_rope_fwd(new[i:i + 1, :, :heads], None, 1e-6, at[i:i + 1], turn)[0][0]
            for h in (0, heads - 1):
                g = h // (heads // kv)
                P.check_forward(o[i, :, h], lse[i, :, h], q[:, h], cache[0, i, :n[i], g], cache[1, i, :n[i], g], True, dim ** -0.5, f"{n} {i} {h}")


@pytest.mark.parametrize("heads,kv_heads,dim,n", [(1, 1, 128, 1), (8, 1, 128, 4), (6, 2, 64, 10), (32, 1, 72, 1), (5, 1, 40, 6), (2, 2, 128, 32)])
@pytest.mark.parametrize("causal", [False, True])
def test_few_queries_of_caches_of_all_lengths(heads, kv_heads, dim, n, causal):
    """Blocks of few rows whose keys end at, before and behind a tile's edge, some with none, in rooms of 1100."""
    used = [0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 600, 1099, 1100]
    room = 1100
    q, k, v = normal((len(used), n, heads, dim), 1), normal((len(used), room, kv_heads, dim), 2), normal((len(used), room, kv_heads, dim), 3)
    for i, m in enumerate(used):   # keys that are not in use may hold anything
        k[i, m:], v[i, m:] = float("nan"), float("inf")
    o, lse = lmbp.attention_fwd(q, k, v, causal, k_lens=torch.tensor(used, device=DEV, dtype=torch.int32))
    group = heads // kv_heads
    for i, m in enumerate(used):
        for h in range(heads):
            P.check_forward(o[i, :, h], lse[i, :, h], q[i, :, h], k[i, :m, h // group], v[i, :m, h // group], causal, dim ** -0.5, f"{m} keys, head {h}")


@pytest.mark.parametrize("tokens,heads,kv_heads,dim", [(1024, 8, 1, 128), (700, 4, 2, 64), (2500, 2, 1, 40)])
def test_many_shares_of_rows(tokens, heads, kv_heads, dim):
    """Few key tiles, whose rows go to as many blocks as fill the device."""
    run(heads, kv_heads, dim, [tokens], [tokens], True)
    run(heads, kv_heads, dim, [tokens - 300, 0, 299, 1], [tokens - 300, 40, 150, 2], False)


def test_frequencies_of_any_size():
    """From denormal numbers to ones whose every position is many turns, of either sign, and those that are whole turns almost."""
    freqs = [5e-324, 1e-300, 2.0 ** -140, 2.0 ** -64, 2.0 ** -63, 1e-12, 1e-4, 0.5, 1.0, -1.0, 3.0, -3.2, 2 * math.pi, -2 * math.pi, 6.5, 1e3, -1e5, 2.0 ** 30, 3e12, -2.0 ** 45, 0.0]
    turn = lmbp.Rotation(freqs)
    x, at = torch.randn(6, 2, 42, device=DEV, generator=torch.Generator(DEV).manual_seed(1)), torch.tensor([1, -1, 2, 7, 0, 1000], device=DEV)
    y, _ = lmbp.rope_fwd(x, None, at, turn)
    t = P.angles(at, turn.freqs, turn.axes, 6)
    want, size = P.turn(x.double(), t, False), P.pair_size(x.double(), 21, False)
    own = torch.cat([t, t], -1).abs() * 2.0 ** -52   # what 64-bit angles themselves are off
    P.inside(y, want, (6 * P.U + own) * size + P.half(torch.float32) * want.abs(), "turned")
    huge = lmbp.Rotation([1e300, -1e18, 2.0 ** 53])   # no angle is meant by these: lengths are kept
    y, _ = lmbp.rope_fwd(x, None, at, huge)
    assert (y.square().sum(-1) - x.square().sum(-1)).abs().max() < 1e-4


# dim, pairs, interleaved: halves that are multiples of 8 bytes and not of 16, for one type or the other, widest ones included
PIECES = [(72, 36, False), (72, 18, False), (24, 12, True), (40, 4, False), (8, 4, False), (4, 2, True), (256, 126, False), (248, 124, False),
          (260, 130, False), (508, 254, False), (504, 252, True), (510, 255, False), (504, 12, False), (12, 0, False), (6, 2, False)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim,pairs,interleaved", PIECES)
def test_heads_in_pieces_of_8_bytes(dim, pairs, interleaved, dtype):
    for tokens, heads, kv_heads in ((70, 5, 2), (9, 17, 1)):
        size = (tokens, heads, kv_heads, dim, pairs, 1, interleaved)
        rope.test_rope(size, dtype)
        for gain in (None, "fp32", "bf16"):
            rope.test_norm_rope(size, gain, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shift", [0, 8, 4, 2])
def test_addresses_of_all_alignments(dtype, shift):
    """The same turn and norm, off by roundings, of heads that lie at multiples of 16, 8, 4 and 2 (4) bytes."""
    step = max(1, shift // dtype.itemsize)
    q = normal((33, 3, 64), 1).to(dtype)
    at, turn = torch.arange(33, device=DEV), lmbp.Rotation.of_base(64)
    room = torch.zeros(33 * 3 * 80 + 64, device=DEV, dtype=dtype)
    here = room[step if shift else 0:][:33 * 3 * 80].view(33, 3, 80)[..., :64]
    here.copy_(q)
    want = lmbp.rope_fwd(q, None, at, turn)[0]
    assert torch.equal(lmbp.rope_fwd(here, None, at, turn)[0], want)
    lmbp.rope_fwd(here, None, at, turn, here)
    assert torch.equal(here, want) and not room.view(-1)[:step if shift else 0].any()
    assert not room[(step if shift else 0):][:33 * 3 * 80].view(33, 3, 80)[..., 64:].any()


def test_keys_are_turned_into_a_cache():
    """k_out may be a row of each sequence's cache; the next call reads it there."""
    room, heads, kv, dim, n = 600, 8, 2, 64, 3
    cache = normal((2, n, room, kv, dim), 1)
    before, turn = cache.clone(), lmbp.Rotation.of_base(dim)
    new = normal((n, 1, heads + 2 * kv, dim), 2)
    q, k, v = new.split((heads, kv, kv), -2)
    at = torch.full((n, 1), 7, device=DEV)
    want = lmbp.rope_fwd(q, k, at, turn)
    yq, yk = lmbp.rope_fwd(q, k, at, turn, k_out=cache[0, :, 7:8])
    cache[1, :, 7:8].copy_(v)
    assert torch.equal(yq, want[0]) and torch.equal(cache[0, :, 7:8], want[1]) and yk.data_ptr() == cache[0, :, 7:8].data_ptr()
    assert torch.equal(cache[0, :, :7], before[0, :, :7]) and torch.equal(cache[0, :, 8:], before[0, :, 8:])
    used = torch.full((n,), 8, device=DEV, dtype=torch.int32)
    o, lse = lmbp.attention_fwd(yq, cache[0], cache[1], True, k_lens=used)
    ref = lmbp.attention_fwd(yq, cache[0, :, :8].contiguous(), cache[1, :, :8].contiguous(), True)
    for i in range(n):
        for h in range(heads):
            P.check_forward(o[i, :, h], lse[i, :, h], yq[i, :, h], cache[0, i, :8, h // 4], cache[1, i, :8, h // 4], True, dim ** -0.5, f"{i} {h}")
            P.check_forward(ref[0][i, :, h], ref[1][i, :, h], yq[i, :, h], cache[0, i, :8, h // 4], cache[1, i, :8, h // 4], True, dim ** -0.5, f"{i} {h}")


def test_gradients_inside_guards():
    """Given outputs between rows of a value of their own: nothing else is written, rows of no sequence stay."""
    rows, heads, kv, dim, lengths = 333, 4, 2, 64, [100, 0, 190, 3]
    used = sum(lengths)
    q, k, v, do = (normal((rows, h, dim), i) for i, h in enumerate((heads, kv, kv, heads)))
    kw = dict(causal=True, q_starts=starts_of(lengths))
    o, lse = lmbp.attention_fwd(q, k, v, **kw)
    want = lmbp.attention_bwd(do, q, k, v, o, lse, **kw)
    room = torch.full((rows + 2, heads + 2 * kv + 1, dim), 7.0, device=DEV, dtype=torch.bfloat16)
    parts = room[1:rows + 1, :heads + 2 * kv].split((heads, kv, kv), 1)
    lmbp.attention_bwd(do, q, k, v, o, lse, dq=parts[0], dk=parts[1], dv=parts[2], **kw)
    for got, ref in zip(parts, want):
        assert torch.equal(got[:used], ref[:used]) and (got[used:] == 7).all() and not ref[used:].any()
    assert (room[0] == 7).all() and (room[-1] == 7).all() and (room[:, -1] == 7).all()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("spare", [0, 5])
def test_more_than_512_sequences(causal, spare):
    """The same as one call per sequence's tokens side by side: lengths of 0 to 3, one of 150, rows of no sequence behind them."""
    lengths = [(5 * i * i + i) % 4 for i in range(1100)]
    lengths[700] = 150
    total = sum(lengths)
    q, k, v, do = (normal((total + spare, h, 64), i) for i, h in enumerate((2, 1, 1, 2)))
    kw = dict(causal=causal, q_starts=starts_of(lengths))
    o, lse = lmbp.attention_fwd(q, k, v, **kw)
    dq, dk, dv = lmbp.attention_bwd(do, q, k, v, o, lse, **kw)
    assert not any(t[total:].any() for t in (o, dq, dk, dv)) and (lse[total:] == -math.inf).all()
    row = 0
    for i, n in enumerate(lengths):
        if n > 0 and (i % 50 < 3 or n > 3 or i > 1080):
            at = slice(row, row + n)
            for h in range(2):
                P.check_forward(o[at, h], lse[at, h], q[at, h], k[at, 0], v[at, 0], causal, 64 ** -0.5, f"sequence {i}")
                parts = P.back_with_room(*(t.double() for t in (do[at, h], q[at, h], k[at, 0], v[at, 0], o[at, h], lse[at, h])), causal, 64 ** -0.5)
                P.inside(dq[at, h], parts[0], parts[3][0] + P.half(torch.bfloat16) * parts[0].abs(), f"sequence {i}: dq")
        row += n
    picked = slice(sum(lengths[:700]), sum(lengths[:701]))   # the long one by itself
    alone = lmbp.attention_fwd(q[picked], k[picked], v[picked], causal)
    assert torch.equal(alone[0], o[picked]) and torch.equal(alone[1], lse[picked])


def test_one_result_given():
    """Where one of o and lse is allocated by the call, rows of no sequence are zeros and -inf in both; with both given they stay."""
    q, k, v = normal((50, 2, 64), 1), normal((50, 2, 64), 2), normal((50, 2, 64), 3)
    kw = dict(q_starts=starts_of([20, 17]))
    want = lmbp.attention_fwd(q, k, v, **kw)
    full = lambda: (torch.full_like(q, 7.0), torch.full((50, 2), 7.0, device=DEV))
    trash = [torch.full((50, 2), 9.0, device=DEV) for _ in range(20)]   # what a new lse may find
    del trash
    for given in ({"o": full()[0]}, {"lse": full()[1]}):
        got = lmbp.attention_fwd(q, k, v, **given, **kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert not got[0][37:].any() and (got[1][37:] == -math.inf).all()
    o, lse = full()
    lmbp.attention_fwd(q, k, v, o=o, lse=lse, **kw)
    assert torch.equal(o[:37], want[0][:37]) and (o[37:] == 7).all() and torch.equal(lse[:37], want[1][:37]) and (lse[37:] == 7).all()
