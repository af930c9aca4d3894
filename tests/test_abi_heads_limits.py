"""Checks on the host of where tensors of heads may lie beside each other, and of the limits of a scale: nothing here
reaches a GPU."""

import ctypes

import pytest
import torch

import paper_2406_16282_amd as lmbp
from paper_2406_16282_amd import binding as B
from test_abi_heads import at, attention, heads, ref, rope


@pytest.fixture(scope="module")
def L():
    return lmbp.lib()


PASSES = B.EHIP   # where there is no GPU to launch on


@pytest.mark.parametrize("rows", [1, 16])
def test_parts_of_the_heads_of_one_tensor_do_not_overlap(L, rows):
    """dq, dk, dv side by side within each head pass, whatever a row's stride is a multiple of; one element more and they meet."""
    if torch.cuda.is_available():
        pytest.skip("a call that passes would launch on addresses that are none")
    a = attention(batch=1, heads=4, kv_heads=4, dim=64, q_rows=rows, k_rows=rows)

    def f(row=12 * 64, head=3 * 64, k_at=64, v_at=128):
        part = lambda off: B._Heads(at(6) + 2 * off, row, head)
        return L.attention_bwd(B.BF16, ref(a), *(ref(heads(i)) for i in range(5)), at(5), ref(part(0)), ref(part(k_at)), ref(part(v_at)),
                               at(9), 1 << 30, None)
    assert f() == f(row=13 * 192) == f(row=16 * 256, head=4 * 64) == f(k_at=128, v_at=64) == PASSES
    assert f(k_at=56) == f(v_at=120) == f(v_at=136) == f(k_at=64 + 192, v_at=64) == B.EOVERLAP
    if rows > 1:
        assert f(row=12 * 64 + 64) == B.EOVERLAP   # the second row's queries lie on the first one's keys

    def turned(q_at=0, k_at=64):
        part = lambda off: B._Heads(at(6) + 2 * off, 8 * 192, 192)
        r = rope(tokens=rows, dim=64, q_heads=8, k_heads=4)
        return L.rope_fwd(B.BF16, ref(r), ref(part(q_at)), ref(part(k_at)), ref(part(q_at)), ref(part(k_at)), None)
    assert turned() == turned(q_at=129) == PASSES   # 129 .. 192 of each head's 192 and 64 .. 127
    assert turned(k_at=63) == turned(q_at=65) == turned(k_at=129, q_at=128) == B.EOVERLAP


def test_the_largest_scale(L):
    """A scale whose product with log2(e) fp32 does not hold makes every score NaN: refused, with no workspace."""
    large = dict(batch=1, q_rows=1, k_rows=65536)
    for scale in (2.4e38, 3.4e38):
        a = attention(scale=scale, **large)
        assert L.attention_fwd(B.BF16, ref(a), ref(heads(0)), ref(heads(1)), ref(heads(2)), ref(heads(3)), at(4), at(5), 1 << 30, None) == B.EINVAL
        assert L.lmbp_attention_fwd_bytes(ref(a)) == L.lmbp_attention_bwd_bytes(ref(a)) == 0
    for scale in (2.3e38, 1e-44):
        assert L.lmbp_attention_fwd_bytes(ref(attention(scale=scale, **large))) > 0
