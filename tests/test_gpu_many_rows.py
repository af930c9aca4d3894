"""More rows, channels or columns than one launch takes (2^32 threads in a grid dimension): narrow
tensors, whose results are compared with those of their halves."""

import ctypes

import pytest
import torch

import paper_2406_16282_amd as lmbp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def same(whole, first, second):
    half = first.shape[0]
    return torch.equal(whole[:half], first) and torch.equal(whole[half:], second)


@pytest.mark.parametrize("cols", [1, 8])
def test_8_bit_rows(cols):
    """Four rows to a block of 256 threads: 2^26 rows and more."""
    rows, half = 2 ** 26 + 5, 2 ** 25
    x = torch.randn(rows, cols, device=DEV).to(torch.bfloat16)
    q, scale = lmbp.q8_rows(x)
    (q0, s0), (q1, s1) = lmbp.q8_rows(x[:half]), lmbp.q8_rows(x[half:])
    assert same(q, q0, q1) and same(scale, s0, s1)
    assert same(lmbp.q8_values(q, scale), lmbp.q8_values(q0, s0), lmbp.q8_values(q1, s1))
    print(f"[q8] rows done {cols}", flush=True)
    del q, scale, q0, s0, q1, s1
    res = torch.randn(rows, cols, device=DEV).to(torch.bfloat16)
    whole = lmbp.msrms_q8_fwd(x, 1e-5, res)
    parts = lmbp.msrms_q8_fwd(x[:half], 1e-5, res[:half]), lmbp.msrms_q8_fwd(x[half:], 1e-5, res[half:])
    assert all(same(w, a, b) for w, a, b in zip(whole, *parts))
    q, scale, rstd, _ = whole
    dx = lmbp.msrms_q8_bwd(x, q, scale, rstd, res)
    assert same(dx, *(lmbp.msrms_q8_bwd(x[p], q[p], scale[p], rstd[p], res[p]) for p in (slice(half), slice(half, None))))


@pytest.mark.parametrize("op", ["msln", "msrms"])
@pytest.mark.parametrize("cols", [1, 8])
def test_norms(op, cols):
    rows, half = 2 ** 26 + 5, 2 ** 25
    fwd, bwd = getattr(lmbp, f"{op}_fwd"), getattr(lmbp, f"{op}_bwd")
    x = torch.randn(rows, cols, device=DEV).to(torch.bfloat16)
    z, rstd = fwd(x, 1e-5)
    (z0, r0), (z1, r1) = fwd(x[:half], 1e-5), fwd(x[half:], 1e-5)
    assert same(z, z0, z1) and same(rstd, r0, r1)
    assert same(bwd(x, z, rstd), bwd(x[:half], z0, r0), bwd(x[half:], z1, r1))


def form(m, n, k, grad=0):
    copies = ctypes.c_int64()
    return lmbp.lib().lmbp_linear_q8_form(m, n, k, grad, None, copies), copies.value


def layer(m, n, k):
    g = torch.Generator(device=DEV).manual_seed(1)
    q = torch.randint(-127, 128, (m, k), generator=g, device=DEV, dtype=torch.int8)
    w = torch.randint(-127, 128, (n, k), generator=g, device=DEV, dtype=torch.int8)
    return q, torch.rand(m, generator=g, device=DEV), w, torch.rand(n, generator=g, device=DEV)


# A row of x against 2^27 and more channels (dot products); as many channels and no product at all
# (the general form); 2^26 and more rows that are copied to aligned ones first.
@pytest.mark.parametrize("m,n,k,kind", [(1, 2 ** 27 + 3, 16, (0, 0)), (1, 2 ** 30 + 5, 0, (8, 0)), (2 ** 26 + 9, 256, 255, (None, 1))])
def test_8_bit_products(m, n, k, kind):
    got = form(m, n, k)
    assert kind[0] in (None, got[0]) and got[1] == kind[1], got
    q, scale, w, w_scale = layer(m, n, k)
    bias = torch.randn(n, device=DEV).to(torch.bfloat16)
    y = lmbp.linear_q8_fwd(q, scale, w, w_scale, bias)
    print(f"[q8] {m} {n} {k} done", flush=True)
    if m == 1:
        for at in range(0, n, 2 ** 24):
            part = slice(at, at + 2 ** 24)
            assert torch.equal(y[:, part], lmbp.linear_q8_fwd(q, scale, w[part], w_scale[part], bias[part]))
        assert k > 0 or torch.equal(y[0], bias)
    else:
        for at in range(0, m, 2 ** 23):
            part = slice(at, at + 2 ** 23)
            assert torch.equal(y[part], lmbp.linear_q8_fwd(q[part], scale[part], w, w_scale, bias))


def test_bias_gradient():
    """A column to a thread, 64 of them to a block: 2^30 columns and more."""
    m, n = 2, 2 ** 30 + 5
    dy = torch.randint(-8, 9, (m, n), device=DEV, dtype=torch.int8).to(torch.bfloat16)
    db = lmbp.linear_bias_grad(dy)
    for at in range(0, n, 2 ** 26):
        assert torch.equal(db[at:at + 2 ** 26], dy[0, at:at + 2 ** 26] + dy[1, at:at + 2 ** 26])


# Flat tensors: 4 values in fp32 to a thread, 2^34 of them and more. One block of values after the other is the
# same; whole tensors in place of their inputs.
BLOCK = 2 ** 20
FLAT = 2 ** 34 + 3 * BLOCK


def repeated(values, n=FLAT):
    t = torch.empty(n, device=DEV)
    t.view(-1, BLOCK).copy_(values.expand(n // BLOCK, BLOCK))
    return t


def repeats(t, values):
    rows = t.view(-1, values.numel())
    return all(bool((rows[i:i + 512] == values).all()) for i in range(0, len(rows), 512))


def room_for(tensors):
    free = torch.cuda.mem_get_info()[0]
    if free < FLAT * 4 * tensors + (24 << 30):
        pytest.skip(f"needs {tensors} tensors of {FLAT * 4 >> 30} GiB, {free >> 30} GiB are free")


@pytest.mark.parametrize("op", ["regelu2", "resilu2"])
def test_activations(op):
    room_for(1)
    fwd, bwd = getattr(lmbp, f"{op}_fwd"), getattr(lmbp, f"{op}_bwd")
    one = torch.randn(BLOCK, device=DEV) * 3
    y, codes = fwd(one)
    x = repeated(one)
    _, many = fwd(x, y=x)
    assert repeats(x, y) and repeats(many, codes)
    bwd(x, many, dx=x)
    assert repeats(x, bwd(y, codes))


@pytest.mark.parametrize("bits", [1, 2, 4])
def test_k_bit_activations(bits):
    room_for(1)
    thresholds = [0.3 * (i - 2 ** (bits - 1)) + 0.1 for i in range(2 ** bits - 1)]
    levels = [0.1 * i - 0.2 for i in range(2 ** bits)]
    one = torch.randn(BLOCK, device=DEV) * 2
    y, codes = lmbp.stepact_fwd(one, "gelu", thresholds, bits)
    x = repeated(one)
    _, many = lmbp.stepact_fwd(x, "gelu", thresholds, bits, y=x)
    assert repeats(x, y) and repeats(many, codes)
    lmbp.stepact_bwd(x, many, levels, bits, dx=x)
    assert repeats(x, lmbp.stepact_bwd(y, codes, levels, bits))


def test_swiglu():
    room_for(3)
    one_g, one_u = torch.randn(BLOCK, device=DEV) * 3, torch.randn(BLOCK, device=DEV)
    h, s, codes = lmbp.reswiglu2_fwd(one_g, one_u)
    g, u = repeated(one_g), repeated(one_u)
    _, many_s, many = lmbp.reswiglu2_fwd(g, u, h=g)
    assert repeats(g, h) and repeats(many_s, s) and repeats(many, codes)
    lmbp.reswiglu2_bwd(g, u, many_s, many, dg=g, du=u)
    dg, du = lmbp.reswiglu2_bwd(h, one_u, s, codes)
    assert repeats(g, dg) and repeats(u, du)


def test_copy():
    room_for(2)
    one = torch.randn(BLOCK, device=DEV)
    src = repeated(one)
    dst = torch.zeros_like(src)
    assert repeats(lmbp.copy_bytes(src, dst), one)
