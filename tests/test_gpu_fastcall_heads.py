"""The native form of the calls on heads (rotary positions, their norms, attention) against the Python path:
the same bytes for the forms that it takes, the Python path's results or errors for those that it declines."""

import pytest

torch = pytest.importorskip("torch")
import paper_2406_16282_amd as lmbp  # noqa: E402
from paper_2406_16282_amd import binding  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Sub(torch.Tensor):
    pass


def randn(*shape, dtype=torch.bfloat16):
    return torch.randn(shape, device=DEV).to(dtype)


def rope_calls():
    torch.manual_seed(0)
    for dtype in (torch.bfloat16, torch.float32):
        fused = randn(2, 5, 3 * 64 * 4, dtype=dtype)
        q, k = (t.unflatten(-1, (-1, 64)) for t in fused.split([8 * 64, 4 * 64], -1))
        at = torch.arange(10, device=DEV)
        turn = lmbp.Rotation.of_base(48)
        yield "rope_fwd", (q, k, at, turn)
        yield "rope_bwd", (q, None, at.int(), turn)
        yield "rope_fwd", (q, k, torch.stack([at, 3 * at]), lmbp.Rotation.of_base(64, sections=(12, 20), interleaved=True))
        yield "rope_fwd", (q, k, torch.stack([at, 3 * at]), turn)
        yield "rope_fwd", (randn(7, 3, 9, dtype=dtype), randn(7, 1, 9, dtype=dtype), at[:7].clone(), lmbp.Rotation((1.0, 0.1)))
        yield "rope_fwd", (q, k, None, lmbp.Rotation(()))
        gains = randn(64), randn(64)
        for gq, gk in ((None, None), gains):
            yq, yk, rq, rk = lmbp.msrms_rope_fwd(q, k, 1e-6, at, turn, gq, gk)
            kept = (yq, yk) if gq is None else (q, k)
            yield "msrms_rope_fwd", (q, k, 1e-6, at, turn, gq, gk)
            yield "msrms_rope_bwd", (q, k, *kept, rq, rk, at, turn, gq, gk)
            yield "msrms_rope_fwd", (q, None, 1e-6, at, turn, gq)
            yield "msrms_rope_bwd", (q, None, kept[0], None, rq, None, at, turn, gq)


def attention_calls():
    torch.manual_seed(0)
    starts = torch.tensor([0, 3, 3, 40], dtype=torch.int32, device=DEV)
    lens = torch.tensor([5, 33], dtype=torch.int32, device=DEV)
    for kwargs, shape, keys in (({}, (2, 33, 4, 64), (2, 33, 2, 64)), ({"causal": True, "scale": 0.2}, (37, 2, 40), (37, 1, 40)),
                                ({"q_starts": starts}, (41, 2, 64), (41, 2, 64)), ({"q_starts": starts, "k_starts": starts}, (41, 2, 128), (40, 1, 128)),
                                ({"k_lens": lens, "causal": True}, (2, 1, 8, 128), (2, 40, 2, 128))):
        q, k, v, do = randn(*shape), randn(*keys), randn(*keys), randn(*shape)
        o, lse = lmbp.attention_fwd(q, k, v, **kwargs)
        yield "attention_fwd", (q, k, v), kwargs
        yield "attention_bwd", (do, q, k, v, o, lse), kwargs
        at = randn(*keys[:-2], 2 * keys[-2], keys[-1]).chunk(2, -2)
        yield "attention_fwd", (q, *at), kwargs


def bits(out):
    out = out if isinstance(out, tuple) else (out,)
    return [None if t is None else (t.dtype, tuple(t.shape), t.stride(), type(t), t.contiguous().view(-1).view(torch.uint8)) for t in out]


def agree(a, b):
    assert len(a) == len(b)
    for x, y in zip(a, b):
        assert (x is None) == (y is None)
        assert x is None or (x[:4] == y[:4] and torch.equal(x[4], y[4]))


def check(op, args, kwargs, monkeypatch):
    lmbp.lib()
    native, took = binding._fast, []

    class Watched:
        def __getattr__(self, name):
            def call(*a):
                out = getattr(native, name)(*a)
                took.append(out is not None)
                return out
            return call

    monkeypatch.setattr(binding, "_fast", Watched())
    got = bits(getattr(lmbp, op)(*args, **kwargs))
    assert took == [True]
    agree(got, bits(getattr(lmbp, op)(*args, **kwargs, stream=torch.cuda.current_stream())))   # the Python path
    assert took == [True]
    agree(got, bits(getattr(lmbp, op)(args[0].as_subclass(Sub), *args[1:], **kwargs)))         # declined
    assert took == [True, False]


def test_rope(monkeypatch):
    for op, args in rope_calls():
        with monkeypatch.context() as m:
            check(op, args, {}, m)


def test_attention(monkeypatch):
    for op, args, kwargs in attention_calls():
        with monkeypatch.context() as m:
            check(op, args, kwargs, m)


def test_given_outputs():
    torch.manual_seed(1)
    q, k, at = randn(6, 4, 32), randn(6, 2, 32), torch.arange(6, device=DEV)
    turn = lmbp.Rotation.of_base(32)
    yq, yk = lmbp.rope_fwd(q, k, at, turn)
    a, b = q.clone(), k.clone()
    out = lmbp.rope_fwd(a, b, at, turn, a, b)
    assert out[0] is a or out[0].data_ptr() == a.data_ptr()
    assert torch.equal(a, yq) and torch.equal(b, yk)
    qkv = randn(2, 9, 3 * 4 * 64)
    q, k, v = (t.unflatten(-1, (4, 64)) for t in qkv.chunk(3, -1))
    o, lse = lmbp.attention_fwd(q, k, v, True)
    want = lmbp.attention_bwd(o, q, k, v, o, lse, True)
    grads = torch.empty_like(qkv)
    parts = [t.unflatten(-1, (4, 64)) for t in grads.chunk(3, -1)]
    lmbp.attention_bwd(o, q, k, v, o, lse, True, dq=parts[0], dk=parts[1], dv=parts[2])
    for got, ref in zip(parts, want):
        assert torch.equal(got, ref)


def test_refusals_come_from_the_python_path():
    q, k, at = randn(6, 4, 32), randn(6, 2, 32), torch.arange(6, device=DEV)
    turn = lmbp.Rotation.of_base(32)
    for error, call in ((ValueError, lambda: lmbp.rope_fwd(q, k, at[:5].clone(), turn)),
                        (TypeError, lambda: lmbp.rope_fwd(q, k, at.float(), turn)),
                        (ValueError, lambda: lmbp.rope_fwd(q, k[:5], at, turn)),
                        (ValueError, lambda: lmbp.rope_fwd(q, k, at, turn, k)),
                        (ValueError, lambda: lmbp.msrms_rope_fwd(q, k, 1e-6, at, turn, randn(32))),
                        (ValueError, lambda: lmbp.attention_fwd(q, k, k[:5])),
                        (ValueError, lambda: lmbp.attention_fwd(q, k, k, q_starts=at)),
                        (TypeError, lambda: lmbp.attention_fwd(q.float(), k, k))):
        with pytest.raises(error):
            call()


def test_the_library_s_refusals():
    q, at = randn(6, 4, 32), torch.arange(6, device=DEV)
    shared = randn(1, 1, 32).expand(6, 4, 32)
    with pytest.raises(lmbp.LmbpError):
        lmbp.rope_fwd(q, None, at, lmbp.Rotation.of_base(32), shared)
    with pytest.raises(lmbp.LmbpError):
        lmbp.attention_fwd(randn(6, 4, 12), randn(6, 4, 12), randn(6, 4, 12))


def test_side_stream():
    q, k, at = randn(64, 8, 128), randn(64, 2, 128), torch.arange(64, device=DEV)
    turn = lmbp.Rotation.of_base(128)
    ref = lmbp.rope_fwd(q, k, at, turn)
    want = lmbp.attention_fwd(*ref, k, True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = lmbp.rope_fwd(q, k, at, turn)
        out = lmbp.attention_fwd(*got, k, True)
    side.synchronize()
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
