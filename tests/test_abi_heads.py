"""Checks on the host of the entry points on tensors of heads (rotation, norm of heads, attention): nothing here
reaches a GPU."""

import copy
import ctypes
import math
import pickle

import pytest
import torch

import paper_2406_16282_amd as lmbp
from paper_2406_16282_amd import binding as B
from paper_2406_16282_amd import nn as lnn

P = 0x7F0000000000   # fake device addresses: every call fails, or is a no-op, before a launch
MiB = 1 << 20


def at(i):
    return P + i * 64 * MiB


def heads(i, row=512, head=64, off=0):
    return B._Heads(at(i) + off, row, head)


def ref(t):
    return None if t is None else ctypes.byref(t)


@pytest.fixture(scope="module")
def L():
    return lmbp.lib()


FREQS = (ctypes.c_double * 32)(*[0.5 ** i for i in range(32)])
BAD = (ctypes.c_double * 32)(*[math.nan] * 32)
AXES = (ctypes.c_int32 * 32)(*[i % 3 for i in range(32)])


def rope(tokens=8, dim=64, q_heads=8, k_heads=4, pairs=32, freqs=FREQS, axes=None, positions=at(9), n_axes=1, wide=1, interleaved=0):
    address = lambda a: None if a is None else ctypes.addressof(a)
    return B._Rope(tokens, dim, q_heads, k_heads, pairs, address(freqs), address(axes), positions, n_axes, wide, interleaved)


@pytest.mark.parametrize("op", ["rope_fwd", "rope_bwd"])
def test_rope(L, op):
    def f(dt=B.BF16, r=rope(), q=heads(0), k=heads(1), yq=heads(2), yk=heads(3)):
        return getattr(L, op)(dt, ref(r), ref(q), ref(k), ref(yq), ref(yk), None)
    assert f(dt=7) == B.EDTYPE
    assert f(r=None) == B.EINVAL
    for bad in (dict(tokens=-1), dict(dim=0), dict(dim=513), dict(q_heads=0), dict(k_heads=-1), dict(pairs=-1), dict(pairs=33),
                dict(n_axes=0), dict(n_axes=256), dict(freqs=None), dict(freqs=BAD), dict(axes=AXES), dict(axes=AXES, n_axes=2),
                dict(positions=None), dict(positions=at(9) + 4), dict(q_heads=1 << 30, dim=64), dict(tokens=1 << 41)):
        assert f(r=rope(**bad)) == B.EINVAL, bad
    assert f(r=rope(tokens=0, positions=None), q=None, k=None, yq=None, yk=None) == B.OK
    assert f(q=None) == f(k=None) == f(yq=None) == f(yk=None) == f(q=B._Heads(None, 512, 64)) == B.EINVAL
    assert f(q=heads(0, off=1)) == f(dt=B.FP32, yq=heads(2, off=2)) == B.EINVAL
    assert f(q=heads(0, row=-8)) == f(k=heads(1, head=-8)) == B.EINVAL
    assert f(yq=heads(2, row=511)) == f(yq=heads(2, head=63)) == f(yq=heads(2, head=0)) == f(yq=heads(2, row=0)) == B.EINVAL
    assert f(yq=heads(0, off=128)) == f(yq=heads(1)) == f(yq=heads(0, row=1024)) == f(yk=heads(2)) == f(yq=heads(9)) == B.EOVERLAP


def test_norm_rope(L):
    def f(dt=B.BF16, dg=B.FP32, r=rope(), eps=1e-5, gq=None, gk=None, q=heads(0), k=heads(1), yq=heads(2), yk=heads(3), sq=at(4), sk=at(5)):
        return L.msrms_rope_fwd(dt, dg, ref(r), eps, gq, gk, ref(q), ref(k), ref(yq), ref(yk), sq, sk, None)
    assert f(dt=7) == f(dg=7) == B.EDTYPE
    assert [f(eps=e) for e in (0.0, -1.0, math.inf, math.nan)] == [B.EINVAL] * 4
    assert f(gq=at(6)) == f(gk=at(6)) == f(gq=at(6), gk=at(7) + 2) == B.EINVAL
    assert f(r=rope(k_heads=0), k=None, yk=None, gk=at(6)) == B.EINVAL
    assert f(sq=None) == f(sk=None) == f(sq=at(4) + 2) == f(q=None) == B.EINVAL
    assert f(r=rope(tokens=0)) == B.OK
    assert f(sq=at(0)) == f(sq=at(2)) == f(sk=at(4)) == f(sk=at(9)) == f(gq=at(2), gk=at(6)) == f(gq=at(4), gk=at(6)) == B.EOVERLAP

    def g(dt=B.BF16, dg=B.FP32, r=rope(), gq=None, gk=None, dq=heads(0), dk=heads(1), q=heads(2), k=heads(3), sq=at(4), sk=at(5),
          xq=heads(6), xk=heads(7), oq=None, ok=None, work=None, size=0):
        return L.msrms_rope_bwd(dt, dg, ref(r), gq, gk, ref(dq), ref(dk), ref(q), ref(k), sq, sk, ref(xq), ref(xk), oq, ok, work, size, None)
    gains = dict(gq=at(10), gk=at(11), oq=at(12), ok=at(13), work=at(14), size=1 << 22)
    assert L.lmbp_msrms_rope_bwd_bytes(64) > 0 and L.lmbp_msrms_rope_bwd_bytes(0) == L.lmbp_msrms_rope_bwd_bytes(513) == 0
    assert g(dt=7) == g(dg=7) == B.EDTYPE
    assert g(sq=None) == g(q=None) == g(xk=None) == g(oq=at(12)) == g(gq=at(10)) == B.EINVAL
    assert g(**dict(gains, oq=None)) == g(**dict(gains, ok=None)) == g(**dict(gains, work=None)) == g(**dict(gains, size=8)) == B.EINVAL
    assert g(**dict(gains, work=at(14) + 8)) == B.EINVAL
    assert g(r=rope(tokens=0)) == B.OK
    assert g(xq=heads(2)) == g(xq=heads(3)) == g(xq=heads(1)) == g(xk=heads(5)) == B.EOVERLAP
    assert g(**dict(gains, oq=at(0))) == g(**dict(gains, oq=at(10))) == g(**dict(gains, ok=at(12))) == g(**dict(gains, work=at(4))) == B.EOVERLAP


def attention(batch=2, heads=8, kv_heads=4, dim=64, q_rows=16, k_rows=16, q_starts=None, k_starts=None, k_lens=None, scale=0.125,
              causal=1, fill=0):
    return B._Attention(batch, heads, kv_heads, dim, q_rows, k_rows, q_starts, k_starts, k_lens, scale, causal, fill)


BAD_PLANS = (dict(batch=0), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(dim=0), dict(dim=12), dict(dim=136), dict(q_rows=-1),
             dict(k_rows=-1), dict(q_rows=17), dict(k_rows=17), dict(q_rows=1 << 31), dict(k_rows=1 << 31),
             dict(q_rows=1 << 30, heads=16), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan),
             dict(q_starts=at(8) + 2), dict(k_lens=at(8) + 1))


def test_attention_fwd(L):
    def f(dt=B.BF16, a=attention(), q=heads(0), k=heads(1), v=heads(2), o=heads(3), lse=at(4), work=None, size=0):
        return L.attention_fwd(dt, ref(a), ref(q), ref(k), ref(v), ref(o), lse, work, size, None)
    assert f(dt=7) == f(dt=B.FP32) == B.EDTYPE
    assert f(a=None) == B.EINVAL
    for bad in BAD_PLANS:
        assert f(a=attention(**bad)) == B.EINVAL, bad
        assert L.lmbp_attention_fwd_bytes(ref(attention(**bad))) == L.lmbp_attention_bwd_bytes(ref(attention(**bad))) == 0
    assert f(a=attention(q_rows=0), q=None, o=None, lse=None) == B.OK
    assert f(q=None) == f(k=None) == f(o=None) == f(lse=None) == f(lse=at(4) + 2) == B.EINVAL
    assert f(q=heads(0, off=8)) == f(k=heads(1, row=516)) == f(v=heads(2, head=68)) == f(o=heads(3, row=504)) == B.EINVAL
    assert f(k=heads(1, row=1 << 23)) == f(q=heads(0, head=1 << 28)) == B.EINVAL
    assert f(o=heads(0)) == f(o=heads(1)) == f(lse=at(3)) == f(lse=at(2)) == B.EOVERLAP
    long = attention(batch=1, q_rows=1, k_rows=65536)
    need = L.lmbp_attention_fwd_bytes(ref(long))
    assert need > 0
    assert f(a=long) == f(a=long, work=at(5), size=need - 1) == f(a=long, work=at(5) + 8, size=need) == B.EINVAL
    assert f(a=long, work=at(1), size=need) == B.EOVERLAP
    starts = attention(q_starts=at(6), k_starts=at(7), k_lens=at(8))
    assert f(a=starts, o=heads(6)) == f(a=starts, lse=at(8)) == B.EOVERLAP


def test_attention_bwd(L):
    def f(dt=B.BF16, a=attention(), do=heads(0), q=heads(1), k=heads(2), v=heads(3), o=heads(4), lse=at(5), dq=heads(6), dk=heads(7),
          dv=heads(8), work=at(9), size=1 << 30):
        return L.attention_bwd(dt, ref(a), ref(do), ref(q), ref(k), ref(v), ref(o), lse, ref(dq), ref(dk), ref(dv), work, size, None)
    assert f(dt=7) == f(dt=B.FP32) == B.EDTYPE
    for bad in BAD_PLANS:
        assert f(a=attention(**bad)) == B.EINVAL, bad
    assert f(a=attention(q_rows=0, k_rows=0), do=None, q=None, k=None, v=None, o=None, lse=None, dq=None, dk=None, dv=None,
             work=None, size=0) == B.OK
    assert f(do=None) == f(lse=None) == f(dq=None) == f(dv=None) == f(work=None) == f(size=16) == f(work=at(9) + 8) == B.EINVAL
    assert f(dk=heads(7, head=32)) == f(dq=heads(6, off=2)) == B.EINVAL
    assert f(dq=heads(1)) == f(dq=heads(0)) == f(dk=heads(8)) == f(dv=heads(4)) == f(dq=heads(5)) == f(work=at(6)) == f(work=at(3)) == B.EOVERLAP


def test_parts_of_one_tensor_do_not_overlap(L):
    """dq, dk, dv as parts of the rows of one tensor pass; one element more and they meet."""
    a = attention(batch=1, heads=8, kv_heads=4, dim=64, q_rows=16, k_rows=16)
    row = (8 + 4 + 4) * 64

    def f(k_at=8 * 64, v_at=12 * 64):
        part = lambda off: B._Heads(at(6) + 2 * off, row, 64)
        return L.attention_bwd(B.BF16, ref(a), ref(heads(0)), ref(heads(1)), ref(heads(2)), ref(heads(3)), ref(heads(4)), at(5),
                               ref(part(0)), ref(part(k_at)), ref(part(v_at)), at(9), 1 << 30, None)
    assert f(k_at=8 * 64 - 8) == f(v_at=12 * 64 - 8) == f(v_at=12 * 64 + 8) == B.EOVERLAP   # the last meets the next row's dq
    if not torch.cuda.is_available():   # the checks pass; there is no GPU to launch on
        assert f() == B.EHIP


def test_rotation():
    r = B.Rotation.of_base(64, sections=(8, 12, 12))
    assert r.n_axes == 3 and len(r.freqs) == 32 and r.freqs[0] == 1.0 and r.axes[8] == 1 and r.axes[31] == 2
    assert abs(B.Rotation.of_base(4, base=100.0).freqs[1] - 0.1) < 1e-15
    for c in (copy.deepcopy(r), pickle.loads(pickle.dumps(r))):
        assert c.freqs == r.freqs and c.axes == r.axes and c._freqs_at != r._freqs_at
    assert B.Rotation(()).freqs == () and B.Rotation.of_base(0).freqs == ()
    for bad in (lambda: B.Rotation([math.inf]), lambda: B.Rotation([1.0], [0, 1]), lambda: B.Rotation([1.0], [-1]),
                lambda: B.Rotation([1.0], [255]), lambda: B.Rotation.of_base(5), lambda: B.Rotation.of_base(8, sections=(1, 2))):
        with pytest.raises(ValueError):
            bad()


def test_binding_refuses_cpu_tensors_and_modules_bad_sizes():
    q, pos, r = torch.zeros(2, 3, 8), torch.zeros(2, dtype=torch.int64), B.Rotation.of_base(8)
    for call in (lambda: lmbp.rope_fwd(q, None, pos, r), lambda: lmbp.rope_bwd(q, None, pos, r),
                 lambda: lmbp.msrms_rope_fwd(q, None, 1e-5, pos, r), lambda: lmbp.attention_fwd(q, q, q),
                 lambda: lmbp.msrms_rope_bwd(q, None, q, None, q, None, pos, r), lambda: lmbp.attention_bwd(q, q, q, q, q, q)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        lmbp.rope_fwd(q, None, pos, [1.0])
    with pytest.raises(ValueError):
        lnn.QKVAttention(8, 3, 64, r)
    with pytest.raises(ValueError):
        lnn.QKVAttention(8, 4, 4, r)
    with pytest.raises(ValueError):
        lnn.QKVAttention(8, 4, 8, r)(torch.zeros(2, 15, 8), pos)
