"""GPU parity of the 8-bit linear layers against products in 64 bits.

With u = 2^-24 and h half a step of the result's type: the sum is exact, its conversion to fp32 u,
the product of the scales u, the multiply-add with the bias u of the result, the store h of it.
The input's gradient: the rows of dy w_scale in 8 bits are those of the oracle exactly; the
conversion, the scale's division and the product u each, the store h.
"""

import ctypes

import pytest
import torch

import paper_2406_16282_amd as lmbp
from paper_2406_16282_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}

# (m, n, k): every remainder of tiles and vectors, single rows and columns, long sums
SIZES = [(3000, 33, 65), (64, 9001, 301), (3, 5, 65), (4, 1, 130), (2, 7, 193), (5, 3, 67), (70, 15, 66), (1, 1, 1), (1, 16, 16), (2, 3, 5), (1, 4096, 512), (3, 1001, 1023), (7, 48, 64), (16, 64, 256), (17, 80, 272),
         (31, 2048, 1040), (33, 24, 48), (64, 130, 257), (65, 1000, 4096), (100, 272, 11008), (127, 255, 129),
         (128, 256, 128), (129, 257, 144), (200, 768, 768), (256, 512, 1024), (257, 528, 1024), (333, 1001, 1023),
         (300, 1003, 4099), (700, 1001, 1023), (1100, 1027, 2051), (20, 100, 4096), (40, 272, 8192), (3000, 272, 272),
         (1100, 2050, 2000), (513, 1040, 2064), (700, 96, 131056), (1000, 8, 32), (1025, 2064, 528), (2100, 4112, 784),
         (2, 33, 2048), (1, 1001, 2064), (2, 13, 4112), (276, 880, 5378), (577, 464, 7414), (347, 809, 7223),
         (130, 784, 6611), (581, 2448, 9527), (2, 13824, 4352)]


def half(t):
    return torch.finfo(t).eps / 2


def weight(n, k, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = torch.randint(-127, 128, (n, k), generator=g, device=DEV, dtype=torch.int8)
    return w, torch.rand(n, generator=g, device=DEV) * 0.01 + 1e-4


def rows(m, k, seed):
    return weight(m, k, seed + 1000)


def bias_of(n, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed + 2000)
    return torch.randn(n, generator=g, device=DEV).to(TYPES[dtype])


def check_fwd(y, q, scale, w, w_scale, bias, what):
    plain = (q.double() @ w.double().t().contiguous()) * scale.double()[:, None] * w_scale.double()
    want = plain if bias is None else plain + bias.double()
    room = 1.01 * (2 * U * plain.abs() + (U + half(y.dtype)) * want.abs()) + 1e-38
    off = (y.double() - want).abs() - room
    assert (off <= 0).all(), f"{what}: {int((off > 0).sum())} values outside, first {(off > 0).nonzero()[0].tolist()}"


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_forward(m, n, k, dtype):
    print(f"[q8] forward {m} {n} {k} {dtype}", flush=True)
    (q, scale), (w, w_scale) = rows(m, k, 1), weight(n, k, 2)
    for bias in (None, bias_of(n, dtype, 3)):
        y = lmbp.linear_q8_fwd(q, scale, w, w_scale, bias, TYPES[dtype])
        assert y.shape == (m, n) and y.dtype == TYPES[dtype]
        check_fwd(y, q, scale, w, w_scale, bias, f"bias {bias is not None}")


def plain_bwd(dy, w, w_scale):
    t = (dy.double() * w_scale.double()).float().double()
    a = t.abs().amax(1).clamp_min(2.0 ** -100)
    p = torch.round(t * (127.0 / a).float().double()[:, None])
    return (p @ w.double()) * (a / 127.0)[:, None], p, a / 127.0


def check_bwd(dx, dy, w, w_scale, what):
    want, _, _ = plain_bwd(dy, w, w_scale)
    room = 1.01 * (3 * U + half(dx.dtype)) * want.abs() + 1e-38
    off = (dx.double() - want).abs() - room
    assert (off <= 0).all(), f"{what}: {int((off > 0).sum())} values outside, first {(off > 0).nonzero()[0].tolist()}"


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_input_gradient(m, n, k, dtype):
    print(f"[q8] input gradient {m} {n} {k} {dtype}", flush=True)
    w, w_scale = weight(n, k, 4)
    g = torch.Generator(device=DEV).manual_seed(5)
    dy = (torch.randn(m, n, generator=g, device=DEV) * 1e-3).to(TYPES[dtype])
    if m > 3:
        dy[1] = 0.0
        dy[2, 0] *= 1000.0
    dx = lmbp.linear_q8_bwd(dy, w, w_scale)
    assert dx.shape == (m, k) and dx.dtype == dy.dtype
    check_bwd(dx, dy, w, w_scale, "dx")
    if m > 3:
        assert (dx[1] == 0).all()
    # against dy times the weight that the layer stands for: half a step of p for every channel
    real = dy.double() @ (w.double() * w_scale.double()[:, None])
    step = (dy.double() * w_scale.double()).abs().amax(1).clamp_min(2.0 ** -100) / 127
    room = (0.5 + 127 * 4 * U) * step[:, None] * w.double().abs().sum(0) + 1.01 * half(dx.dtype) * (dx.double().abs() + real.abs())
    assert ((dx.double() - real).abs() <= room + 1e-5 * real.abs() + 1e-38).all()


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32"), ("fp32", "bf16")])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_input_gradients_that_add_up(m, n, k, dtype, out):
    """dx = product + add with one rounding (u of the sum in the multiply-add, h in the store)."""
    w, w_scale = weight(n, k, 4)
    dy = (torch.randn(m, n, device=DEV) * 1e-3).to(TYPES[dtype])
    add = torch.randn(m, k, device=DEV).to(TYPES[out])
    part, _, _ = plain_bwd(dy, w, w_scale)
    want = part + add.double()
    dx = lmbp.linear_q8_bwd(dy, w, w_scale, add)
    assert dx.dtype == TYPES[out]
    room = 1.01 * (3 * U * part.abs() + (U + half(dx.dtype)) * want.abs()) + 1e-38
    assert ((dx.double() - want).abs() <= room).all()
    assert torch.equal(lmbp.linear_q8_bwd(dy, w, w_scale, add, dx=add), dx) and torch.equal(add, dx)   # in place
    assert lmbp.linear_q8_bwd(dy, w, w_scale, dtype=TYPES[out]).dtype == TYPES[out]


LARGE = [(4096, 4096, 2048), (2048, 11008, 4096), (300, 4096, 11008), (20, 11008, 4096), (40, 13824, 1024), (400, 4096, 4096),
         (1000, 8208, 2064), (1000, 2064, 8208), (40, 4112, 4112), (70, 8208, 2064), (100, 1040, 4112)]


@pytest.mark.parametrize("m,n,k", LARGE)
def test_large_layers(m, n, k):
    (q, scale), (w, w_scale) = rows(m, k, 6), weight(n, k, 7)
    check_fwd(lmbp.linear_q8_fwd(q, scale, w, w_scale), q, scale, w, w_scale, None, "forward")
    dy = torch.randn(m, n, device=DEV).to(torch.bfloat16)
    check_bwd(lmbp.linear_q8_bwd(dy, w, w_scale), dy, w, w_scale, "gradient")


def forms(grad, sizes):
    shares, copies = ctypes.c_int64(), ctypes.c_int64()
    for m, n, k in sizes:
        yield lmbp.lib().lmbp_linear_q8_form(m, n, k, grad, shares, copies), shares.value, copies.value


def test_the_sizes_take_every_form():
    fwd = set(forms(0, SIZES + LARGE))
    assert {f for f, _, _ in fwd} == set(range(9)) and {c for _, _, c in fwd} == {0, 1}, fwd
    bwd = set(forms(1, [(m, n, k) for m, k, n in SIZES] + LARGE))
    assert {f for f, _, _ in bwd} == set(range(1, 9)) and {c for _, _, c in bwd} == {0, 1}, bwd
    assert {s for f, s, _ in bwd if f <= 3} >= {1, 2, 4, 8}, bwd
    assert {s for f, s, _ in bwd if f == 4} >= {1, 2, 4, 8}, bwd


@pytest.mark.parametrize("m,n,k", [(1, 32, 131071), (70, 64, 131056), (3, 9, 131071)])
def test_the_longest_sums_are_exact(m, n, k):
    """-128 in every place: the sum is 2^31 - 2^14 at most, and its fp32 value is what comes out."""
    q = torch.full((m, k), -128, dtype=torch.int8, device=DEV)
    w = torch.full((n, k), -128, dtype=torch.int8, device=DEV)
    w[n // 2] = 127
    y = lmbp.linear_q8_fwd(q, torch.ones(m, device=DEV), w, torch.ones(n, device=DEV), dtype=torch.float32)
    want = torch.full((n,), 16384.0 * k, device=DEV, dtype=torch.float64)
    want[n // 2] = -128.0 * 127.0 * k
    assert torch.equal(y, want.float().expand(m, n))


@pytest.mark.parametrize("m,k", [(5, 64), (200, 272), (17, 33)])
def test_no_products_and_nothing_to_do(m, k):
    n = 48
    bias = bias_of(n, "fp32", 1)
    none = torch.empty(0, dtype=torch.int8, device=DEV)
    scale, w_scale = torch.rand(m, device=DEV), torch.rand(n, device=DEV)
    y = lmbp.linear_q8_fwd(none.view(m, 0), scale, none.view(n, 0), w_scale, bias, torch.float32)
    assert torch.equal(y, bias.expand(m, n))
    assert (lmbp.linear_q8_fwd(none.view(m, 0), scale, none.view(n, 0), w_scale) == 0).all()
    dx = lmbp.linear_q8_bwd(torch.empty(m, 0, device=DEV), none.view(0, k), torch.empty(0, device=DEV))
    assert dx.shape == (m, k) and (dx == 0).all()
    w, w_scale = weight(n, k, 1)
    assert lmbp.linear_q8_fwd(none.view(0, k), scale[:0], w, w_scale).shape == (0, n)
    assert lmbp.linear_q8_bwd(torch.empty(0, n, device=DEV), w, w_scale).shape == (0, k)


@pytest.mark.parametrize("m,n,k", [(1, 64, 64), (200, 272, 1024), (9, 33, 65)])
def test_rows_that_are_not_finite_stay_by_themselves(m, n, k):
    m += 2
    (q, scale), (w, w_scale) = rows(m, k, 1), weight(n, k, 2)
    clean = lmbp.linear_q8_fwd(q, scale, w, w_scale)
    scale[1] = float("nan")
    y = lmbp.linear_q8_fwd(q, scale, w, w_scale)
    assert y[1].isnan().all()
    keep = [i for i in range(m) if i != 1]
    assert torch.equal(y[keep], clean[keep])
    dy = torch.randn(m, n, device=DEV)
    clean = lmbp.linear_q8_bwd(dy, w, w_scale)
    dy[1, n // 2] = float("inf")
    dx = lmbp.linear_q8_bwd(dy, w, w_scale)
    assert dx[1].isnan().all() and torch.equal(dx[keep], clean[keep])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m,n,k,shift", [(5, 64, 64, 1), (200, 272, 512, 3), (33, 100, 160, 1), (130, 257, 1024, 2)])
def test_any_address_and_nothing_beside_the_result(m, n, k, shift, dtype):
    t = TYPES[dtype]

    def band(src=None, count=0, kind=None):
        count, kind = (src.numel(), src.dtype) if src is not None else (count, kind)
        buf = torch.full((count + 64,), 77, dtype=kind, device=DEV)
        view = buf[16 + shift:16 + shift + count]
        if src is not None:
            view.copy_(src.reshape(-1))
        return buf, view, ctypes.c_void_p(view.data_ptr())

    def whole(b):
        return bool((b[0][:16 + shift] == 77).all() and (b[0][16 + shift + b[1].numel():] == 77).all())

    (q, scale), (w, w_scale), bias = rows(m, k, 1), weight(n, k, 2), bias_of(n, dtype, 3)
    bq, bs, bw, bws, bb = band(q), band(scale), band(w), band(w_scale), band(bias)
    by, bdx = band(count=m * n, kind=t), band(count=m * k, kind=t)
    dy = torch.randn(m, n, device=DEV).to(t)
    bdy = band(dy)
    L, dt = lmbp.lib(), B.BF16 if dtype == "bf16" else B.FP32
    st = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert L.lmbp_linear_q8_fwd_bytes(m, n, k) == 0
    assert L.linear_q8_fwd(dt, m, n, k, bq[2], bs[2], bw[2], bws[2], bb[2], by[2], None, 0, st) == B.OK
    assert torch.equal(by[1].view(m, n), lmbp.linear_q8_fwd(q, scale, w, w_scale, bias, t))
    need = L.lmbp_linear_q8_bwd_bytes(m, n, k)
    work = torch.full((need + 64,), 77, dtype=torch.uint8, device=DEV)
    assert L.linear_q8_bwd(dt, dt, m, n, k, bdy[2], bw[2], bws[2], None, bdx[2], ctypes.c_void_p(work.data_ptr()), need, st) == B.OK
    assert torch.equal(bdx[1].view(m, k), lmbp.linear_q8_bwd(dy, w, w_scale))
    torch.cuda.synchronize()
    assert all(whole(b) for b in (bq, bs, bw, bws, bb, by, bdx, bdy)) and (work[need:] == 77).all()


def test_results_behind_the_2_31st_value():
    m, n, k = 140_000, 16_400, 64
    (q, scale), (w, w_scale) = rows(m, k, 1), weight(n, k, 2)
    y = lmbp.linear_q8_fwd(q, scale, w, w_scale)
    for part in (slice(0, 64), slice(130_900, 131_200), slice(m - 100, m)):
        check_fwd(y[part], q[part], scale[part], w, w_scale, None, str(part))
    del y
    m, n, k = 140_000, 64, 16_400
    w, w_scale = weight(n, k, 3)
    dy = torch.randn(m, n, device=DEV).to(torch.bfloat16)
    dx = lmbp.linear_q8_bwd(dy, w, w_scale)
    for part in (slice(0, 64), slice(130_900, 131_200), slice(m - 100, m)):
        check_bwd(dx[part], dy[part], w, w_scale, str(part))


def test_inputs_behind_the_2_31st_byte():
    m, n, k = 66_000, 32, 32_768
    w, w_scale = weight(n, k, 1)
    q = torch.zeros(m, k, dtype=torch.int8, device=DEV)
    at = [0, 65_535, 65_536, m - 1]
    some, _ = rows(4, k, 2)
    q[at] = some
    scale = torch.ones(m, device=DEV)
    y = lmbp.linear_q8_fwd(q, scale, w, w_scale)
    assert torch.equal(y[at], lmbp.linear_q8_fwd(some, scale[:4], w, w_scale)) and (y[1:65_535] == 0).all()
    # as the weight: 66 000 channels
    y = lmbp.linear_q8_fwd(some, scale[:4], q, scale)
    assert torch.equal(y[:, at], lmbp.linear_q8_fwd(some, scale[:4], some, scale[:4])) and (y[:, 1:65_535] == 0).all()
    dy = torch.randn(3, m, device=DEV).to(torch.bfloat16)
    check_bwd(lmbp.linear_q8_bwd(dy, q[:, :64].contiguous(), scale), dy, q[:, :64].contiguous(), scale, "long sums")


@pytest.mark.parametrize("m,n,k,what", [(333, 1001, 1023, "copies"), (16, 11008, 512, "shares")])
def test_two_graphs_at_once_with_workspaces(m, n, k, what):
    """Two graphs of one size, each with workspaces of its own, replayed on two streams at the same
    time, with eager calls between: every replay against the eager result."""
    shares, copies = ctypes.c_int64(), ctypes.c_int64()
    lmbp.lib().lmbp_linear_q8_form(m, n, k, 1, shares, copies)
    assert copies.value == 1 if what == "copies" else shares.value > 1
    w, w_scale = weight(n, k, 1)

    def run(q, scale, dy):
        return lmbp.linear_q8_fwd(q, scale, w, w_scale), lmbp.linear_q8_bwd(dy, w, w_scale)

    ins = [[*rows(m, k, s), torch.randn(m, n, device=DEV)] for s in (2, 3)]
    for i in ins:
        run(*i)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in ins:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(run(*i))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in graphs]
    for replay in range(4):
        for q, _, dy in ins:
            q.random_(-127, 128)
            dy.normal_()
        want = [run(*i) for i in ins]
        for o in outs:
            for v in o:
                v.fill_(7.0)
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        run(*ins[0])
        torch.cuda.synchronize()
        for o, v in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(o, v)), f"replay {replay}"


@pytest.mark.parametrize("m,n,k", [(333, 1001, 1023), (16, 11008, 512)])
def test_workspaces_on_another_stream(m, n, k):
    """The stream argument: what the default stream allocates next is not the launch's workspace."""
    (q, scale), (w, w_scale) = rows(m, k, 1), weight(n, k, 2)
    dy = torch.randn(m, n, device=DEV)
    want = lmbp.linear_q8_fwd(q, scale, w, w_scale), lmbp.linear_q8_bwd(dy, w, w_scale)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(4):
        got = (lmbp.linear_q8_fwd(q, scale, w, w_scale, stream=side), lmbp.linear_q8_bwd(dy, w, w_scale, stream=side))
        for nbytes in (1 << 16, 1 << 20, 1 << 22, 1 << 24):
            torch.full((nbytes,), 255, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_shapes_and_refusals():
    (q, scale), (w, w_scale) = rows(6, 32, 1), weight(48, 32, 2)
    y = lmbp.linear_q8_fwd(q.view(2, 3, 32), scale.view(2, 3), w, w_scale)
    assert y.shape == (2, 3, 48) and torch.equal(y.view(6, 48), lmbp.linear_q8_fwd(q, scale, w, w_scale))
    dx = lmbp.linear_q8_bwd(y, w, w_scale)
    assert dx.shape == (2, 3, 32)
    cases = [
        (ValueError, lambda: lmbp.linear_q8_fwd(q.float(), scale, w, w_scale)),
        (ValueError, lambda: lmbp.linear_q8_fwd(q, scale, w.float(), w_scale)),
        (ValueError, lambda: lmbp.linear_q8_fwd(q, scale, w.t(), w_scale)),
        (ValueError, lambda: lmbp.linear_q8_fwd(q[:, :16].contiguous(), scale, w, w_scale)),
        (ValueError, lambda: lmbp.linear_q8_fwd(q, scale[:3], w, w_scale)),
        (ValueError, lambda: lmbp.linear_q8_fwd(q, scale.double(), w, w_scale)),
        (ValueError, lambda: lmbp.linear_q8_fwd(q, scale, w, w_scale[:3])),
        (ValueError, lambda: lmbp.linear_q8_fwd(q, scale, w, w_scale, bias_of(48, "fp32", 1))),
        (ValueError, lambda: lmbp.linear_q8_fwd(q, scale, w, w_scale, bias_of(32, "bf16", 1))),
        (TypeError, lambda: lmbp.linear_q8_fwd(q, scale, w, w_scale, dtype=torch.float16)),
        (ValueError, lambda: lmbp.linear_q8_fwd(q, scale, w.view(-1), w_scale)),
        (TypeError, lambda: lmbp.linear_q8_bwd(y.half(), w, w_scale)),
        (ValueError, lambda: lmbp.linear_q8_bwd(y[..., :16].contiguous(), w, w_scale)),
        (ValueError, lambda: lmbp.linear_q8_bwd(y, w, w_scale.bfloat16())),
        (ValueError, lambda: lmbp.linear_q8_bwd(y.transpose(0, 1), w, w_scale)),
        (ValueError, lambda: lmbp.linear_q8_bwd(y, w, w_scale, add=dx[:1])),
        (ValueError, lambda: lmbp.linear_q8_bwd(y, w, w_scale, add=dx, dx=dx.float())),
        (TypeError, lambda: lmbp.linear_q8_bwd(y, w, w_scale, dtype=torch.float16)),
    ]
    for error, call in cases:
        with pytest.raises(error):
            call()
    long = torch.zeros(2, 131_072, dtype=torch.int8, device=DEV)
    with pytest.raises(lmbp.LmbpError):
        lmbp.linear_q8_fwd(long, scale[:2], long, scale[:2])
