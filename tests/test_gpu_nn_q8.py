"""The 8-bit modules: the operators run together as a model runs them, forward and backward,
on other streams, in graphs, and what they keep for the backward."""

import pytest
import torch

import paper_2406_16282_amd as lmbp
from paper_2406_16282_amd.nn import (LinearQ8, MSRMSNormLinearQ8, ReSwiGLU2, merge_norm_into_linears)

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


def layer(n, k, seed, bias=False, dtype=torch.float32):
    torch.manual_seed(seed)
    lin = torch.nn.Linear(k, n, bias=bias, device=DEV, dtype=dtype)
    return lin, LinearQ8.from_linear(lin)


def rows64(t):
    a = t.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -100)
    return torch.round(t * (127.0 / a).float().double()), a


def linear64(x, mod):
    """The layer on the rows of x in 8 bits, in 64 bits (the sums are whole numbers, so exact)."""
    q, a = rows64(x)
    return product64(q, a / 127.0, mod)


def product64(q, scale, mod):
    y = (q @ mod.weight.double().t().contiguous()) * scale * mod.scale.double()
    return y if mod.bias is None else y + mod.bias.double()


def back64(dy, mod):
    t = (dy.double() * mod.scale.double()).float().double()
    p, a = rows64(t)
    return (p @ mod.weight.double()) * (a / 127.0)


@pytest.mark.parametrize("bias", [False, True])
def test_linear_module(bias):
    lin, mod = layer(272, 144, 1, bias)
    # the weight is the layer's up to half a scale per channel
    assert ((mod.values(torch.float32) - lin.weight).abs() <= (0.5 + 1e-4) * mod.scale[:, None]).all()
    x = torch.randn(2, 37, 144, device=DEV, requires_grad=True)
    if bias:
        mod.bias.requires_grad_()
    y = mod(x)
    want = linear64(x.detach().double().view(-1, 144), mod).view(2, 37, 272)
    size = want.abs() + (mod.bias.abs().double() if bias else 0.0)
    assert ((y - want).abs() <= 8 * U * size + 1e-38).all()
    kept = y.grad_fn.saved_tensors
    assert {t.data_ptr() for t in kept} == {mod.weight.data_ptr(), mod.scale.data_ptr()}   # nothing of x
    dy = torch.randn_like(y)
    y.backward(dy)
    dx = back64(dy.view(-1, 272), mod).view_as(x)
    assert ((x.grad - dx).abs() <= 4 * U * dx.abs() + 1e-38).all()
    if bias:   # 74 values to a sum
        db = dy.double().sum((0, 1))
        assert ((mod.bias.grad - db).abs() <= 76 * U * dy.double().abs().sum((0, 1))).all()


@pytest.mark.parametrize("with_res", [False, True])
@pytest.mark.parametrize("rows,k,sizes", [(50, 144, (272, 16, 96)), (1, 64, (40,)), (33, 77, (50, 61))])
def test_norm_and_layers(rows, k, sizes, with_res):
    mods = [layer(n, k, 3 + i, bias=i == 1)[1] for i, n in enumerate(sizes)]
    block = MSRMSNormLinearQ8(mods, eps=1e-5)
    torch.manual_seed(7)
    x = torch.randn(rows, k, device=DEV, requires_grad=True)
    res = torch.randn(rows, k, device=DEV, requires_grad=True) if with_res else None
    out = block(x, res)
    out = out if isinstance(out, tuple) else (out,)
    assert len(out) == len(sizes) + int(with_res)
    s = (x + res if with_res else x).detach()
    if with_res:
        assert torch.equal(out[-1], s)
    s64 = s.double()
    eps32 = float(torch.tensor(1e-5, dtype=torch.float32))
    rstd = (s64.square().mean(-1, keepdim=True) + eps32).rsqrt()
    q, a = rows64(s64)
    z = q * (a * rstd / 127.0)
    for y, mod in zip(out, mods):
        want = product64(q, a * rstd / 127.0, mod)
        # rstd by c = k / 64 + 24 additions and 6 roundings, then the layer's
        assert ((y - want).abs() <= ((k / 64 + 24) / 2 + 10) * U * (
            want.abs() + (mod.bias.abs().double() if mod.bias is not None else 0.0))).all()
    dys = [torch.randn_like(y) for y in out]
    torch.autograd.backward(out, dys)
    parts = [back64(dy, mod) for dy, mod in zip(dys, mods)]
    dz = sum(parts)
    along = (z * dz).mean(-1, keepdim=True)
    want = rstd * (dz - z * along) + (dys[-1].double() if with_res else 0.0)
    # dz off by 5 u of its parts; z and rstd by those of above; the norm's own sum and roundings
    e = sum(p.abs() for p in parts) * (5 + len(parts)) * U
    c = (k / 64 + 24) * 2 + 20
    room = rstd * (e + z.abs() * (z.abs() * e).mean(-1, keepdim=True)) + c * U * (
        rstd * (dz.abs() + z.abs() * (z * dz).abs().mean(-1, keepdim=True)) + want.abs())
    assert ((x.grad - want).abs() <= 1.01 * room).all()
    if with_res:
        assert torch.equal(res.grad, x.grad)


def test_outputs_that_are_not_used():
    mods = [layer(n, 64, n)[1] for n in (48, 32)]
    block = MSRMSNormLinearQ8(mods)
    x, res = (torch.randn(9, 64, device=DEV, requires_grad=True) for _ in range(2))
    y0, y1, s = block(x, res)
    g, = torch.autograd.grad(s.sum(), x, retain_graph=True)
    assert torch.equal(g, torch.ones_like(g))
    dy = torch.randn_like(y1)
    g, = torch.autograd.grad(y1, res, dy, retain_graph=True)
    q, scale, rstd = lmbp.msrms_q8_fwd((x + res).detach(), block.eps)
    dz = lmbp.linear_q8_bwd(dy, mods[1].weight, mods[1].scale, dtype=torch.float32)
    assert torch.equal(g, lmbp.msrms_q8_bwd(dz, q, scale, rstd))
    x2 = x.detach()
    assert block(x2)[0].grad_fn is None and block(x2, res)[2].requires_grad
    with torch.no_grad():
        assert all(torch.equal(a, b) for a, b in zip(block(x, res), (y0, y1, s)))


def test_what_a_block_keeps():
    """One byte per element and two numbers per row, for the norm and its layers together."""
    rows, k = 256, 512
    block = MSRMSNormLinearQ8([layer(256, k, 1, dtype=torch.bfloat16)[1], layer(64, k, 2, dtype=torch.bfloat16)[1]])
    x = torch.randn(rows, k, device=DEV, dtype=torch.bfloat16, requires_grad=True)
    y, _ = block(x)
    own = {t.data_ptr() for t in block.buffers()}
    kept = [t for t in y.grad_fn.saved_tensors if t.data_ptr() not in own]
    assert sum(t.numel() * t.element_size() for t in kept) == rows * k + 8 * rows


def mlp(k, f, dtype):
    """A LLaMA MLP block in 8 bits: norm, gate and up, SwiGLU, down."""
    torch.manual_seed(11)
    norm = torch.nn.RMSNorm(k, eps=1e-5, device=DEV, dtype=dtype)
    with torch.no_grad():
        norm.weight.uniform_(0.5, 1.5)
    lins = [torch.nn.Linear(k, f, bias=False, device=DEV, dtype=dtype) for _ in range(2)]
    merge_norm_into_linears(norm, lins)
    down = torch.nn.Linear(f, k, bias=False, device=DEV, dtype=dtype)
    first = MSRMSNormLinearQ8([LinearQ8.from_linear(m) for m in lins], eps=1e-5)
    return first, ReSwiGLU2(), LinearQ8.from_linear(down)


def step(parts, x, res, dy, ds):
    first, act, down = parts
    g, u, s = first(x, res)
    y = down(act(g, u))
    return y, s, *torch.autograd.grad((y, s), (x, res), (dy, ds))


def test_mlp_block_step_by_step():
    """The block through autograd against the entry points called one after the other."""
    k, f, rows = 256, 688, 70
    parts = mlp(k, f, torch.bfloat16)
    x, res = (torch.randn(rows, k, device=DEV, dtype=torch.bfloat16, requires_grad=True) for _ in range(2))
    dy, ds = (torch.randn(rows, k, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    y, s, dx, dres = step(parts, x, res, dy, ds)
    first, _, down = parts
    gate, up = first.layers
    q, sc, rstd, s1 = lmbp.msrms_q8_fwd(x.detach(), 1e-5, res.detach())
    g, u = (lmbp.linear_q8_fwd(q, sc, m.weight, m.scale) for m in (gate, up))
    h, act, codes = lmbp.reswiglu2_fwd(g, u)
    hq, hs = lmbp.q8_rows(h)
    y1 = lmbp.linear_q8_fwd(hq, hs, down.weight, down.scale)
    dh = lmbp.linear_q8_bwd(dy, down.weight, down.scale)
    dg, du = lmbp.reswiglu2_bwd(dh, u, act, codes)
    dz = lmbp.linear_q8_bwd(dg, gate.weight, gate.scale, dtype=torch.float32)
    dz = lmbp.linear_q8_bwd(du, up.weight, up.scale, add=dz)
    dx1 = lmbp.msrms_q8_bwd(dz, q, sc, rstd, ds)
    for got, want in ((y, y1), (s, s1), (dx, dx1), (dres, dx1)):
        assert torch.equal(got, want)


def test_mlp_block_near_the_block_that_it_stands_for():
    """fp32: the block with 8-bit rows is within the rounding to 8 bits of the one without.
    Each product's operands are off by half a step of their row, 1/254 of its largest value:
    with 256 to 688 terms of random signs a relative error of about 1/254 * max / rms * sqrt(1/3)
    each, 4 operands on the way: 0.04 leaves twice that (max / rms is 3.5 here)."""
    k, f, rows = 256, 688, 70
    first, act, down = mlp(k, f, torch.float32)
    x = torch.randn(rows, k, device=DEV)
    g, u = first(x)
    y = down(act(g, u)).double()
    z = x.double() * (x.double().square().mean(-1, keepdim=True) + 1e-5).rsqrt()
    wg, wu, wd = (m.weight.double() * m.scale.double()[:, None] for m in (*first.layers, down))
    g64, u64 = z @ wg.t().contiguous(), z @ wu.t().contiguous()
    want = (torch.nn.functional.silu(g64) * u64) @ wd.t().contiguous()
    assert ((y - want).norm() / want.norm()) <= 0.04


@pytest.mark.parametrize("rows", [1, 70, 400])
def test_graph_of_the_block(rows):
    """Forward and backward captured, two graphs at a time, replayed with new inputs and eager
    work between; every replay against the eager result."""
    k, f = 256, 688
    parts = mlp(k, f, torch.bfloat16)
    first, _, down = parts
    gate, up = first.layers

    def run(x, res, dy, ds):
        q, sc, rstd, s = lmbp.msrms_q8_fwd(x, 1e-5, res)
        g, u = (lmbp.linear_q8_fwd(q, sc, m.weight, m.scale) for m in (gate, up))
        h, act, codes = lmbp.reswiglu2_fwd(g, u)
        hq, hs = lmbp.q8_rows(h)
        y = lmbp.linear_q8_fwd(hq, hs, down.weight, down.scale)
        dh = lmbp.linear_q8_bwd(dy, down.weight, down.scale)
        dg, du = lmbp.reswiglu2_bwd(dh, u, act, codes)
        dz = lmbp.linear_q8_bwd(dg, gate.weight, gate.scale, dtype=torch.float32)
        dz2 = lmbp.linear_q8_bwd(du, up.weight, up.scale, add=dz)
        return y, s, dz2, lmbp.q8_values(q, sc), lmbp.msrms_q8_bwd(dz2, q, sc, rstd, ds)

    ins = [[torch.randn(rows, k, device=DEV).to(torch.bfloat16) for _ in range(4)] for _ in range(2)]
    for i in ins:
        run(*i)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in ins:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(*i))
        graphs.append(g)
    for replay in range(3):
        for i in ins:
            for t in i:
                t.normal_()
        want = [run(*i) for i in ins]
        torch.cuda.synchronize()
        for o in outs:
            for t in o:
                t.view(torch.uint8).fill_(0xA5)
        for n in ((0, 1), (1, 0), (0, 1))[replay]:
            graphs[n].replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(o, w)), f"replay {replay}"


def test_captured_training_step():
    """The modules' forward and backward in one graph. The eager steps have leaves of their own and
    their graphs are gone before the capture; every replay against an eager step."""
    parts = mlp(256, 688, torch.bfloat16)
    ins = [torch.randn(130, 256, device=DEV, dtype=torch.bfloat16) for _ in range(4)]

    def eager():
        x, res, dy, ds = (v.clone() for v in ins)
        return [v.detach() for v in step(parts, x.requires_grad_(), res.requires_grad_(), dy, ds)]

    eager()
    torch.cuda.synchronize()
    x, res = (v.clone().requires_grad_() for v in ins[:2])
    dy, ds = (v.clone() for v in ins[2:])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = [v.detach() for v in step(parts, x, res, dy, ds)]
    for replay in range(3):
        with torch.no_grad():
            for v, to in zip(ins, (x, res, dy, ds)):
                v.normal_()
                to.copy_(v)
            for v in out:
                v.fill_(7.0)
        want = eager()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), f"replay {replay}"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n", [(130, 272), (20011, 48), (6000, 1024), (100000, 16), (70000, 1)])
def test_captured_bias_gradients(rows, n, dtype):
    """The biases' gradients, sums over all rows, in a graph. Of small whole numbers, so that every
    order of additions in fp32 is exact: every replay against the sum in 64 bits."""
    torch.manual_seed(5)
    mod = LinearQ8.from_linear(torch.nn.Linear(64, n, device=DEV, dtype=dtype))
    mod.bias.requires_grad_()
    x = torch.randn(rows, 64, device=DEV, dtype=dtype)
    dy = torch.randint(-8, 9, (rows, n), device=DEV).to(dtype)
    torch.autograd.grad(mod(x), mod.bias, dy)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        db, = torch.autograd.grad(mod(x), mod.bias, dy)
    for replay in range(4):
        dy.copy_(torch.randint(-8, 9, (rows, n), device=DEV))
        eager, = torch.autograd.grad(mod(x), mod.bias, dy)
        db.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        want = dy.double().sum(0).to(dtype)
        assert torch.equal(db, want) and torch.equal(eager, want), f"replay {replay}"


def test_on_another_stream():
    parts = mlp(256, 688, torch.bfloat16)
    x, res = (torch.randn(200, 256, device=DEV, dtype=torch.bfloat16, requires_grad=True) for _ in range(2))
    dy, ds = (torch.randn(200, 256, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    want = step(parts, x, res, dy, ds)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step(parts, x, res, dy, ds)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    down = parts[2]
    side.wait_stream(torch.cuda.current_stream())
    for handle in (side, side.cuda_stream):      # the entry points' own stream argument
        q, sc, rstd, s = lmbp.msrms_q8_fwd(x.detach(), 1e-5, res.detach(), stream=handle)
        y = lmbp.linear_q8_fwd(q, sc, parts[0].layers[0].weight, parts[0].layers[0].scale, stream=handle)
        dx = lmbp.linear_q8_bwd(dy, down.weight, down.scale, stream=handle)
        side.synchronize()
        q1, sc1, rstd1, s1 = lmbp.msrms_q8_fwd(x.detach(), 1e-5, res.detach())
        assert torch.equal(q, q1) and torch.equal(sc, sc1) and torch.equal(rstd, rstd1) and torch.equal(s, s1)
        assert torch.equal(y, lmbp.linear_q8_fwd(q1, sc1, parts[0].layers[0].weight, parts[0].layers[0].scale))
        assert torch.equal(dx, lmbp.linear_q8_bwd(dy, down.weight, down.scale))


def test_two_threads_on_two_streams():
    """Calls made at the same time by two host threads, each on a stream of its own."""
    import threading
    torch.manual_seed(3)
    (_, mod) = layer(1001, 1023, 1)
    xs = [torch.randn(130, 1023, device=DEV) for _ in range(2)]
    dys = [torch.randn(130, 1001, device=DEV) for _ in range(2)]

    def run(x, dy):
        q, scale, rstd = lmbp.msrms_q8_fwd(x, 1e-5)
        dz = lmbp.linear_q8_bwd(dy, mod.weight, mod.scale)
        return lmbp.linear_q8_fwd(q, scale, mod.weight, mod.scale), lmbp.msrms_q8_bwd(dz, q, scale, rstd)

    want = [run(x, dy) for x, dy in zip(xs, dys)]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(20):
                got = run(xs[i], dys[i])
                s.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                    bad.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not bad


@pytest.mark.parametrize("shape", [(0, 144), (2, 0, 144), (144,), (1, 1, 144)])
def test_modules_of_no_rows_and_of_one(shape):
    (_, a), (_, b) = layer(272, 144, 1, True), layer(33, 144, 2)
    a.bias.requires_grad_()
    x, res = (torch.randn(shape, device=DEV, requires_grad=True) for _ in range(2))
    block = MSRMSNormLinearQ8([a, b])
    ya, yb, s = block(x, res)
    assert ya.shape == (*shape[:-1], 272) and yb.shape == (*shape[:-1], 33) and s.shape == x.shape
    (ya.sum() + yb.sum() + s.sum() + a(x).sum()).backward()      # gradients that are expanded numbers
    assert x.grad.shape == x.shape and res.grad.shape == x.shape
    rows = x.numel() // 144
    assert torch.equal(a.bias.grad, torch.full((272,), 2.0 * rows, device=DEV))
    q, scale, rstd, s1 = lmbp.msrms_q8_fwd(x.detach(), block.eps, res.detach())
    dz = lmbp.linear_q8_bwd(torch.ones_like(ya), a.weight, a.scale)
    dz = lmbp.linear_q8_bwd(torch.ones_like(yb), b.weight, b.scale, add=dz)
    assert torch.equal(res.grad, lmbp.msrms_q8_bwd(dz, q, scale, rstd, torch.ones_like(s1)))
    if rows == 0:
        assert x.grad.numel() == 0


def test_one_layer_twice_and_frozen_inputs():
    (_, a) = layer(48, 64, 1, True)
    a.bias.requires_grad_()
    x = torch.randn(9, 64, device=DEV)
    y0, y1 = MSRMSNormLinearQ8([a, a])(x)
    assert torch.equal(y0, y1)
    d0, d1 = torch.randn_like(y0), torch.randn_like(y1)
    torch.autograd.backward((y0, y1), (d0, d1))       # no input asks for a gradient, the bias does
    want = (d0.double() + d1.double()).sum(0)
    assert ((a.bias.grad - want).abs() <= 20 * U * (d0.abs() + d1.abs()).double().sum(0)).all()


def test_the_same_twice():
    """No result depends on the order in which blocks run."""
    (_, mod), x = layer(1040, 2064, 1), torch.randn(300, 2064, device=DEV)
    q, s, r = lmbp.msrms_q8_fwd(x, 1e-5)
    dy = torch.randn(300, 1040, device=DEV)
    first = None
    for _ in range(3):
        out = (lmbp.linear_q8_fwd(q, s, mod.weight, mod.scale, dtype=torch.float32), lmbp.linear_q8_bwd(dy, mod.weight, mod.scale),
               *lmbp.msrms_q8_fwd(x, 1e-5), lmbp.msrms_q8_bwd(x, q, s, r))
        first = first or out
        assert all(torch.equal(a, b) for a, b in zip(out, first))


def calls(shape, dtype):
    torch.manual_seed(0)
    here = torch.cuda.current_stream()
    x, res, dz, ds = (torch.randn(shape, device=DEV).to(dtype) for _ in range(4))
    q, scale, rstd = lmbp.msrms_q8_fwd(x, 1e-5, stream=here)
    w = torch.randint(-127, 128, (33, shape[-1]), device=DEV, dtype=torch.int8)
    w_scale, bias = torch.rand(33, device=DEV), torch.randn(33, device=DEV).to(dtype)
    dy = torch.randn(*shape[:-1], 33, device=DEV).to(dtype)
    yield lmbp.q8_rows, (x,), {}
    yield lmbp.q8_values, (q, scale), {}
    yield lmbp.q8_values, (q, scale, dtype), {}
    yield lmbp.msrms_q8_fwd, (x, 1e-5), {}
    yield lmbp.msrms_q8_fwd, (x, 1e-5, res), {}
    yield lmbp.msrms_q8_bwd, (dz, q, scale, rstd), {}
    yield lmbp.msrms_q8_bwd, (dz, q, scale, rstd, ds), {}
    yield lmbp.msrms_q8_bwd, (dz.float(), q, scale, rstd), {"dtype": dtype}
    yield lmbp.linear_q8_fwd, (q, scale, w, w_scale, None, dtype), {}
    yield lmbp.linear_q8_fwd, (q, scale, w, w_scale, bias, dtype), {}
    yield lmbp.linear_q8_bwd, (dy, w, w_scale), {}
    yield lmbp.linear_q8_bwd, (dy, w, w_scale), {"dtype": torch.float32}
    yield lmbp.linear_q8_bwd, (dy, w, w_scale, res), {}


class Sub(torch.Tensor):
    pass


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(1,), (3, 40), (2, 5, 64), (0, 16), (7, 1023)])
def test_native_calls_and_the_python_path(shape, dtype):
    """The same results from the native form of a call, from the Python path (a stream given) and
    from a call that the native form declines (a subclass)."""
    from paper_2406_16282_amd import binding
    lmbp.lib()
    assert binding._fast is not None
    for op, args, more in calls(shape, dtype):
        outs = (op(*args, **more), op(*args, **more, stream=torch.cuda.current_stream()),
                op(args[0].as_subclass(Sub), *args[1:], **more))
        outs = [o if isinstance(o, tuple) else (o,) for o in outs]
        for a, b, c in zip(*outs):
            assert type(a) is torch.Tensor and a.shape == b.shape and a.dtype == b.dtype and a.stride() == b.stride()
            assert torch.equal(a.reshape(-1).view(torch.uint8), b.reshape(-1).view(torch.uint8)), op.__name__
            assert torch.equal(b.reshape(-1).view(torch.uint8), c.reshape(-1).view(torch.uint8)), op.__name__
