"""Modules of rotation and attention on the GPU: gradients through autograd, a whole attention block, graphs, streams."""

import math

import pytest
import torch
from torch import nn

import paper_2406_16282_amd as lmbp
import plain_heads as P
from paper_2406_16282_amd import binding as B
from paper_2406_16282_amd import nn as lnn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5


def normal(shape, seed, std=1.0, dtype=torch.bfloat16):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def starts_of(lengths):
    return torch.tensor([0, *lengths], device=DEV).cumsum(0).int()


def rel(got, want):
    return ((got.double() - want.double()).norm() / want.double().norm()).item()


def plain_heads(x, pos, r, eps=None, gain=None):
    """Rotation (norm, gain) of [rows, heads, dim] in 64 bits, through autograd."""
    t = P.angles(pos, r.freqs, r.axes, x.shape[0])
    if eps is not None:
        x = P.norm(x, eps)[0]
    return P.turn(x if gain is None else x * gain, t, r.interleaved)


def plain_attention(q, k, v, lengths, causal):
    """Packed attention in 64 bits, through autograd."""
    group = q.shape[1] // k.shape[1]
    out, row = [], 0
    for n in lengths:
        a = slice(row, row + n)
        out.append(torch.stack([P.attend(q[a, h], k[a, h // group], v[a, h // group], causal, q.shape[2] ** -0.5)[0]
                                for h in range(q.shape[1])], 1))
        row += n
    return torch.cat(out)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gains", [False, True])
def test_rope_and_norm_rope_gradients(dtype, gains):
    """Through autograd against 64 bits: inside a few roundings of the type (y is rounded, and starts the backward)."""
    r = B.Rotation.of_base(48, sections=(8, 8, 8))
    pos = torch.randint(0, 500, (3, 70), device=DEV)
    q, k = normal((70, 6, 64), 1, dtype=dtype).requires_grad_(), normal((70, 2, 64), 2, dtype=dtype).requires_grad_()
    dq, dk = normal((70, 6, 64), 3, dtype=dtype), normal((70, 2, 64), 4, dtype=dtype)
    q64, k64 = (t.detach().double().requires_grad_() for t in (q, k))
    limit = 4 * torch.finfo(dtype).eps
    yq, yk = lnn.Rope(r)(q, k, pos)
    got = torch.autograd.grad((yq, yk), (q, k), (dq, dk))
    want = torch.autograd.grad((plain_heads(q64, pos, r), plain_heads(k64, pos, r)), (q64, k64), (dq.double(), dk.double()))
    assert all(rel(a, b) < limit for a, b in zip(got, want))
    (only,) = torch.autograd.grad(lnn.Rope(r)(q, k, pos)[1], k, dk)   # one of the two
    assert torch.equal(only, got[1])

    m = lnn.MSRMSNormRope(r, EPS, 64 if gains else None, DEV)
    if gains:
        with torch.no_grad():
            m.q_gain.copy_(normal((64,), 5, dtype=torch.float32)), m.k_gain.copy_(normal((64,), 6, dtype=torch.float32))
    params = list(m.parameters())
    ws = [p.detach().double().requires_grad_() for p in params] or [None, None]
    yq, yk = m(q, k, pos)
    got = torch.autograd.grad((yq, yk), (q, k, *params), (dq, dk))
    ref = plain_heads(q64, pos, r, EPS, ws[0]), plain_heads(k64, pos, r, EPS, ws[1])
    want = torch.autograd.grad(ref, (q64, k64, *(w for w in ws if w is not None)), (dq.double(), dk.double()))
    assert rel(yq, ref[0]) < limit and rel(yk, ref[1]) < limit
    assert all(rel(a, b) < limit for a, b in zip(got, want))


@pytest.mark.parametrize("causal", [False, True])
def test_attention_gradients(causal):
    lengths = [60, 1, 130]
    q, k, v, do = (normal((191, h, 64), i) for i, h in enumerate((6, 2, 2, 6)))
    leaves = [t.requires_grad_() for t in (q, k, v)]
    s = starts_of(lengths)
    o = lnn.Attention(causal)(q, k, v, s)
    got = torch.autograd.grad(o, leaves, do)
    l64 = [t.detach().double().requires_grad_() for t in leaves]
    ref = plain_attention(*l64, lengths, causal)
    want = torch.autograd.grad(ref, l64, do.double())
    assert rel(o, ref) < 0.01 and all(rel(a, b) < 0.01 for a, b in zip(got, want))   # P, dS and o: a rounding each
    # transposed heads (rows not one behind the other) and an expanded gradient are taken, by copies where they must be
    q2 = q.detach().transpose(0, 1).contiguous().transpose(0, 1).requires_grad_()
    o2 = lnn.Attention(causal)(q2, k, v, s)
    assert torch.equal(o2, o)
    o2.sum().backward()
    assert q2.grad.shape == q2.shape


@pytest.mark.parametrize("eps", [None, EPS])
@pytest.mark.parametrize("form", ["dense", "packed"])
def test_qkv_attention(form, eps):
    lengths = [50, 50, 50] if form == "dense" else [20, 100, 1, 29]
    heads, kv_heads, dim = 6, 2, 64
    r = B.Rotation.of_base(64)
    rows = sum(lengths) + (7 if form == "packed" else 0)   # rows of no sequence
    qkv = normal((rows, heads + 2 * kv_heads, dim), 1).requires_grad_()
    pos = torch.cat([torch.arange(n, device=DEV) for n in lengths] + [torch.zeros(rows - sum(lengths), device=DEV, dtype=torch.int64)])
    do = normal((rows, heads, dim), 2)
    m = lnn.QKVAttention(heads, kv_heads, dim, r, eps=eps)
    if form == "dense":
        o = m(qkv.view(3, 50, -1, dim), pos.view(3, 50)).flatten(0, 1)
    else:
        o = m(qkv, pos, starts_of(lengths))
    (got,) = torch.autograd.grad(o, qkv, do)
    n = sum(lengths)
    x = qkv.detach().double().requires_grad_()
    q, k, v = x[:n].split((heads, kv_heads, kv_heads), 1)
    ref = plain_attention(plain_heads(q, pos[:n], r, eps), plain_heads(k, pos[:n], r, eps), v, lengths, True)
    (want,) = torch.autograd.grad(ref, x, do[:n].double())
    assert rel(o[:n], ref) < 0.01 and rel(got, want) < 0.015   # the turned q and k are rounded besides
    assert (o[n:] == 0).all() and (got[n:] == 0).all()
    # the same as its parts one behind the other
    q, k, v = (t.detach().requires_grad_() for t in qkv.split((heads, kv_heads, kv_heads), 1))
    y = lnn.Rope(r)(q, k, pos) if eps is None else lnn.MSRMSNormRope(r, eps)(q, k, pos)
    parts = lnn.Attention(True)(*y, v, starts_of(lengths))
    grads = torch.autograd.grad(parts, (q, k, v), do)
    assert torch.equal(parts, o) and torch.equal(torch.cat(grads, 1), got)


class Block(nn.Module):
    """Norm, projections, attention, output projection of a block, with the residual."""

    def __init__(self, width, heads, kv_heads):
        super().__init__()
        self.dim = width // heads
        self.norm = lnn.MSRMSNorm(EPS)
        self.qkv = nn.Linear(width, (heads + 2 * kv_heads) * self.dim, bias=False, device=DEV, dtype=torch.bfloat16)
        self.attention = lnn.QKVAttention(heads, kv_heads, self.dim, B.Rotation.of_base(self.dim), eps=EPS)
        self.out = nn.Linear(width, width, bias=False, device=DEV, dtype=torch.bfloat16)

    def forward(self, x, positions, starts=None):
        y = self.qkv(self.norm(x)).unflatten(-1, (-1, self.dim))
        return x + self.out(self.attention(y, positions, starts).flatten(-2))


def test_block_trains():
    """A block with the operators together: gradients against torch's operations in 32 bits, and a few steps."""
    torch.manual_seed(0)
    block = Block(256, 4, 2)
    x = normal((2, 90, 256), 1).requires_grad_()
    pos = torch.arange(90, device=DEV).expand(2, 90)
    dy = normal((2, 90, 256), 2)
    y = block(x, pos)
    got = torch.autograd.grad(y, (x, block.qkv.weight, block.out.weight), dy)
    x64, w, u = (t.detach().double().requires_grad_() for t in (x, block.qkv.weight, block.out.weight))
    h = (P.norm(x64, EPS)[0] @ w.t()).view(180, 8, 64)
    q, k, v = h.split((4, 2, 2), 1)
    r, flat = block.attention.rotation, pos.reshape(-1).contiguous()
    o = plain_attention(plain_heads(q, flat, r, EPS), plain_heads(k, flat, r, EPS), v, [90, 90], True)
    ref = x64 + (o.flatten(1) @ u.t()).view(2, 90, 256)
    want = torch.autograd.grad(ref, (x64, w, u), dy.double())
    assert rel(y, ref) < 0.02 and all(rel(a, b) < 0.03 for a, b in zip(got, want))   # five roundings to bf16 on the way
    opt = torch.optim.SGD(block.parameters(), lr=0.1)
    for _ in range(3):
        opt.zero_grad()
        (block(x, pos).float() - dy.float()).square().mean().backward()
        opt.step()
    assert all(p.isfinite().all() and p.grad.isfinite().all() for p in block.parameters())


def test_what_is_kept():
    """QKVAttention keeps the turned queries and keys, qkv's storage (its values), the output and a value per row."""
    rows, heads, kv_heads, dim = 128, 4, 2, 64
    qkv = normal((rows, heads + 2 * kv_heads, dim), 1).requires_grad_()
    pos = torch.arange(rows, device=DEV)
    kept = {}
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.setdefault(t.untyped_storage().data_ptr(), t) is None or t, lambda t: t):
        lnn.QKVAttention(heads, kv_heads, dim, B.Rotation.of_base(dim), eps=EPS)(qkv, pos)
    size = sum(t.untyped_storage().nbytes() for p, t in kept.items() if p not in (qkv.untyped_storage().data_ptr(), pos.untyped_storage().data_ptr()))
    assert size == rows * ((heads + kv_heads) * dim * 2 + heads * dim * 2 + heads * 4 + (heads + kv_heads) * 4)


def steps(qkv, pos, s, do, module):
    o = module(qkv, pos, s)
    (d,) = torch.autograd.grad(o, qkv, do)
    return o.detach(), d


def test_captured_and_replayed():
    """Forward and backward in a graph, replayed on other inputs between eager calls: the eager results. The starts are read
    on the device, so other sequences of the same sum are taken."""
    heads, kv_heads, dim, rows = 8, 2, 128, 300
    qkv, do = normal((rows, heads + 2 * kv_heads, dim), 1).requires_grad_(), normal((rows, heads, dim), 2)
    pos, s = torch.arange(rows, device=DEV), starts_of([100, 200])
    m = lnn.QKVAttention(heads, kv_heads, dim, B.Rotation.of_base(dim), eps=EPS)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        steps(qkv, pos, s, do, m)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = steps(qkv, pos, s, do, m)
    for i, lengths in enumerate(([100, 200], [1, 299], [250, 50], [150, 150])):
        with torch.no_grad():
            qkv.copy_(normal(qkv.shape, 10 + i))
        s.copy_(starts_of(lengths))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = steps(qkv, pos, s, do, m)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), lengths


def test_two_graphs_with_workspaces():
    """Two captured forwards whose keys are split, replayed on two streams at once: each has its workspace."""
    k, v = normal((20000, 2, 128), 1), normal((20000, 2, 128), 2)
    qs = [normal((1, 8, 128), i) for i in (3, 4)]
    want = [lmbp.attention_fwd(q, k, v) for q in qs]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for q in qs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(lmbp.attention_fwd(q, k, v))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for (o, lse), (a, b) in zip(outs, want):
            assert torch.equal(o, a) and torch.equal(lse, b)
            o.zero_(), lse.zero_()
        torch.cuda.synchronize()


def test_other_streams():
    """A stream given, a raw handle, and torch's current one: the same results, the workspace on the launch's stream."""
    q, do = normal((40, 16, 64), 1), normal((40, 16, 64), 2)
    k, v = normal((900, 1, 64), 3), normal((900, 1, 64), 4)
    r, pos = B.Rotation.of_base(64), torch.arange(40, device=DEV)
    w = torch.randn(64, device=DEV)
    f = lambda **s: [*lmbp.attention_fwd(q, k, v, causal=True, **s)]
    b = lambda o, lse, **s: [*lmbp.attention_bwd(do, q, k, v, o, lse, causal=True, **s)]
    n = lambda **s: [t for t in lmbp.msrms_rope_fwd(q, None, EPS, pos, r, w, **s) if t is not None]
    g = lambda rstd, **s: [t for t in lmbp.msrms_rope_bwd(do, None, q, None, rstd, None, pos, r, w, **s) if t is not None]
    o, lse = f()
    y = n()
    want = [o, lse, *b(o, lse), *y, *g(y[1])]
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    for s in (dict(stream=st), dict(stream=st.cuda_stream)):
        got = [*f(**s), *b(o, lse, **s), *n(**s), *g(y[1], **s)]
        st.synchronize()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, want))
    with torch.cuda.stream(st):
        got = [*f(), *b(o, lse), *n(), *g(y[1])]
    st.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, want))


def test_under_autocast():
    r, pos = B.Rotation.of_base(64), torch.arange(30, device=DEV)
    qkv = normal((30, 6, 64), 1).requires_grad_()
    m = lnn.QKVAttention(2, 2, 64, r)
    o = m(qkv, pos)
    (d,) = torch.autograd.grad(o, qkv, o.detach())
    with torch.autocast("cuda", torch.float16):
        o2 = m(qkv, pos)
        (d2,) = torch.autograd.grad(o2, qkv, o2.detach())
    assert torch.equal(o, o2) and torch.equal(d, d2)
    with pytest.raises(TypeError):
        m(qkv.float(), pos)
