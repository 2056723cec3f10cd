"""Int8 projections on the GPU (readings Q1-Q3): codes and scales bit for bit
where they come from the inputs themselves, within the rounding of fp32 behind
RMSNorm and the gate; products bit for bit without a residual, every tile of the
dispatch and every kind of K tail among the sizes."""
import numpy as np
import pytest
import torch

from gpu_helpers import log
from oracle import bf16_round
from oracle import int8 as Q
from paper_2609_04875_amd import gemm_int8, gemm_int8_multi, quantize_rows, rmsnorm_int8, silu_mul_int8

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _bf(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().to(BF)


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


ROWS = [(1, 16), (3, 48), (7, 1232), (2, 2048), (5, 2064), (300, 4096), (257, 8192), (4, 14336), (300, 18944),
        (2, 32768), (3, 36000), (2, 133136), (1, 4112)]


@pytest.mark.parametrize("m,k", ROWS)
@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_rows_bit_exact(m, k, dtype):
    log(f"quantize_rows {m} x {k} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(k)
    x = torch.randn(m, k, device="cuda", generator=g) * torch.exp(3 * torch.randn(m, 1, device="cuda", generator=g))
    if m > 2:
        x[0] = 0
        x[1, k // 2] = float("nan")
        x[2, k - 1] = float("-inf")
    x = x.to(dtype)
    q, s = quantize_rows(x)
    wq, ws = Q.quantize_rows(x.float().cpu().numpy())
    assert np.array_equal(q.cpu().numpy(), wq) and np.array_equal(s.cpu().numpy(), ws, equal_nan=True)


def test_rows_of_subnormals_and_of_the_largest():
    x = torch.zeros(4, 64, device="cuda")
    x[0, :3] = torch.tensor([2.0 ** -149, -2.0 ** -148, 0])
    x[1, :3] = torch.tensor([200 * 2.0 ** -149, -1 * 2.0 ** -149, 80 * 2.0 ** -149])
    x[2, :3] = torch.tensor([3.4e38, -1.7e38, 1e30])
    x[3, 5] = -1e-30
    q, s = quantize_rows(x)
    wq, ws = Q.quantize_rows(x.cpu().numpy())
    assert np.array_equal(q.cpu().numpy(), wq) and np.array_equal(s.cpu().numpy(), ws)


def _check_codes(q, s, y, slack):
    """Codes of fp64 values y: y_i / s = 127 y_i / max |y| is known to ``slack``
    relative roundings of fp32, so a code is off its value by a half and that."""
    top = np.abs(y).max(-1)
    assert (np.abs(s - top / 127) <= 1e-5 * top / 127).all()
    exact = 127 * y / top[:, None]
    assert (np.abs(q - exact) <= 0.5 + 127 * slack * 2.0 ** -24).all()


@pytest.mark.parametrize("m,k", ROWS)
def test_rmsnorm_rows(m, k):
    log(f"rmsnorm_int8 {m} x {k}")
    rng = np.random.default_rng(k)
    x, gain = bf16_round(rng.standard_normal((m, k)) * 3), bf16_round(1 + 0.1 * rng.standard_normal(k))
    q, s = rmsnorm_int8(_bf(x), _bf(gain), 1e-5)
    # gain, factor, scale, quotient of the element and of the largest
    _check_codes(q.cpu().numpy(), s.cpu().numpy().astype(np.float64), Q.rmsnorm(x, gain, 1e-5), 8)


@pytest.mark.parametrize("m,k", ROWS)
def test_gate_rows(m, k):
    log(f"silu_mul_int8 {m} x {k}")
    rng = np.random.default_rng(k)
    gu = bf16_round(rng.standard_normal((m, 2 * k)) * 3)
    q, s = silu_mul_int8(_bf(gu))
    # the exponential to 2 roundings, sum, quotient, product, scale, quotient; element and largest
    _check_codes(q.cpu().numpy(), s.cpu().numpy().astype(np.float64), Q.silu_mul(gu), 20)


def test_rows_that_are_not_finite():
    x = torch.ones(5, 32, dtype=BF, device="cuda")
    x[1, 3], x[2, 4], x[3], x[4, 0] = float("nan"), float("inf"), 0, 1e30       # its square leaves fp32
    gain = torch.ones(32, dtype=BF, device="cuda")
    q, s = rmsnorm_int8(x, gain, 0.0)
    s = s.cpu().numpy()
    assert s[0] > 0 and np.isnan(s[1:]).all() and not q[1:].any()
    q, s = rmsnorm_int8(x, gain, 1e-5)
    assert s[3] == 0 and not q[3].any()
    gu = torch.ones(3, 64, dtype=BF, device="cuda")
    gu[1, 3], gu[2, 40] = float("-inf"), float("nan")
    q, s = silu_mul_int8(gu)
    assert torch.isfinite(s[0]) and torch.isnan(s[1:]).all() and not q[1:].any()
    wq, ws = quantize_rows(torch.ones(8, 32, dtype=BF, device="cuda"))
    y = gemm_int8(q, s, wq, ws)
    assert torch.isfinite(y[0]).all() and torch.isnan(y[1:]).all()


def test_gates_far_from_zero():
    """SiLU of gates from the smallest to the largest: 0 far below, the gate itself
    far above; a row of far negative gates is a row of zeros."""
    g = torch.tensor([-3e38, -1e30, -1000.0, -126.0, -88.0, -87.0, -60.0, -20.0, -1e-30, 0.0, 1e-30, 20.0, 90.0, 1000.0,
                      -0.0, 3e-39], dtype=torch.float64)
    for gate in (g, g.clamp(max=-90.0), g.clamp(max=-50.0), g.clamp(max=1.0), g.clamp(max=1e-30)):
        gu = torch.cat([gate, torch.ones(16, dtype=torch.float64)])[None].to(BF).cuda()
        q, s = silu_mul_int8(gu)
        y = Q.silu_mul(np.maximum(_np(gu), -700.0))
        y[np.abs(y) < 2.0 ** -119] = 0                  # below what the kernel keeps
        top = np.abs(y).max()
        if top == 0:
            assert s.item() == 0 and not q.any()
        else:
            _check_codes(q.cpu().numpy(), s.cpu().numpy().astype(np.float64), y, 40)


def test_sizes_past_32_bits():
    """x, w and y each of more than 2^31 elements, their last rows and columns against
    products of those alone."""
    log("x of 2.3e9 codes")
    m, k, n = 140008, 16400, 8
    x = torch.zeros(m, k, dtype=torch.int8, device="cuda")
    part = torch.randint(-127, 128, (300, k), dtype=torch.int8, device="cuda")
    x[-300:] = part
    s, ws = torch.rand(m, device="cuda") + 0.5, torch.rand(n, device="cuda") + 0.5
    w = torch.randint(-127, 128, (n, k), dtype=torch.int8, device="cuda")
    y = gemm_int8(x, s, w, ws)
    assert torch.equal(y[-300:], gemm_int8(part, s[-300:].clone(), w, ws)) and not y[:-300].any()
    log("w of 2.3e9 codes")
    y = gemm_int8(w[:3].contiguous(), s[:3].contiguous(), x, s)
    assert torch.equal(y[:, -304:], gemm_int8(w[:3].contiguous(), s[:3].contiguous(), x[-304:], s[-304:].clone()))
    assert not y[:, :-304].any()
    del x, y
    log("rows of 2.3e9 values")
    x = torch.zeros(m, k, dtype=BF, device="cuda")
    x[-2:] = torch.randn(2, k, device="cuda").to(BF)
    q, sc = quantize_rows(x)
    q2, s2 = quantize_rows(x[-2:].contiguous())
    assert torch.equal(q[-2:], q2) and torch.equal(sc[-2:], s2) and not q[-9:-2].any() and not sc[:-2].any()
    del x, q
    log("y of 4.4e9 values")
    m = n = 66000
    x, w = torch.zeros(m, 16, dtype=torch.int8, device="cuda"), torch.zeros(n, 16, dtype=torch.int8, device="cuda")
    x[-5:], w[-9:] = 3, 2
    one = torch.ones(m, device="cuda")
    y = gemm_int8(x, one, w, one)
    assert (y[-5:, -9:] == 96).all() and not y[-5:, :-9].any() and not y[-6].any() and not y[0].any()


def test_more_rows_than_one_launch():
    m = (1 << 21) + 3
    x = torch.ones(m, 16, dtype=BF, device="cuda")
    x[-2, 3] = -2
    q, s = quantize_rows(x)
    assert (q[:-2] == 127).all() and q[-2, 3] == -127 and q[-2, 0] == 64 and (s[:-2] == s[0]).all() and (q[-1] == 127).all()


def _operands(m, n, k, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    xq = torch.randint(-127, 128, (m, k), generator=g, dtype=torch.int8, device="cuda")
    wq = torch.randint(-127, 128, (n, k), generator=g, dtype=torch.int8, device="cuda")
    return xq, torch.rand(m, device="cuda", generator=g) + 0.1, wq, torch.rand(n, device="cuda", generator=g) + 0.1


def _sum(xq, wq):
    return torch.matmul(xq.double(), wq.double().t().contiguous())         # exact: below 2^53


def _want(xq, xs, wq, ws):
    """fp32(sum) * (xs * ws) rounded to bf16: fp32(sum) of an integer is one rounding, as the kernel's."""
    return (_sum(xq, wq).float() * (xs[:, None] * ws)).to(BF)


PRODUCTS = [(1, 8, 16), (1, 4096, 4096), (2, 1024, 144), (3, 16, 32), (16, 24, 48), (17, 40, 112), (31, 1000, 128),
            (33, 264, 240), (64, 512, 256), (65, 2056, 272), (102, 3584, 18944), (128, 128, 384), (129, 136, 1232),
            (300, 4104, 4112), (333, 1000, 1232), (1000, 1000, 1008), (1025, 2048, 2064), (2048, 4096, 512),
            (2049, 4104, 528), (4096, 8192, 1024), (4100, 8200, 656), (70000, 8, 16), (5, 128256, 64), (1, 8, 133136),
            (9, 20008, 4112), (40, 200, 8208), (201, 3592, 1168), (700, 8200, 1152), (2049, 2056, 2176), (16, 16392, 1024),
            (7, 3592, 18960), (27, 3592, 2064), (190, 4104, 2064), (33, 4104, 8208), (280, 3592, 8208)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product_bit_exact(m, n, k):
    log(f"gemm_int8 {m} x {n} x {k}")
    xq, xs, wq, ws = _operands(m, n, k, m + n + k)
    y = gemm_int8(xq, xs, wq, ws)
    assert torch.equal(y, _want(xq, xs, wq, ws))
    r = torch.randn(m, n, device="cuda").to(BF)
    out = r.clone()
    gemm_int8(xq, xs, wq, ws, r=out, out=out)                               # in place, as a residual is added
    exact = _sum(xq, wq) * (xs.double()[:, None] * ws.double())
    want = exact + r.double()
    # one rounding to bf16 of a sum of fp32 terms, each within three fp32 roundings
    bound = 2.0 ** -8 * want.abs() + 3 * 2.0 ** -24 * (exact.abs() + r.double().abs())
    assert ((out.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("k", [16, 512, 2048, 2064, 4096, 8192, 8208, 18944])
def test_quantised_rows_do_not_depend_on_the_others(k):
    """A row's codes and scale in calls of 1, 256, 257 and 2000 rows, bit for bit."""
    log(f"rows of {k} in calls of different sizes")
    x = (torch.randn(2000, 2 * k, device="cuda") * 3).to(BF)
    gain = (torch.randn(k, device="cuda") * 0.3 + 1).to(BF)
    for f, y in ((lambda t: rmsnorm_int8(t, gain, 1e-5), x[:, :k].contiguous()), (silu_mul_int8, x),
                 (quantize_rows, x[:, k:].contiguous()), (quantize_rows, x[:, k:].float().contiguous())):
        q, s = f(y)
        for m in (1, 256, 257):
            q2, s2 = f(y[300:300 + m])
            assert torch.equal(q2, q[300:300 + m]) and torch.equal(s2, s[300:300 + m]), m


@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_residual_bit_exact(m, n, k):
    """The product with the scales, then the addition, each rounded to fp32, whatever
    kernel the size takes: a row's bits depend on its own operands alone."""
    log(f"gemm_int8 with residual {m} x {n} x {k}")
    xq, xs, wq, ws = _operands(m, n, k, m + n + k)
    y = _sum(xq, wq).float() * (xs[:, None] * ws)
    r = (y * torch.rand(m, n, device="cuda")).to(BF)             # of the product's own size
    assert torch.equal(gemm_int8(xq, xs, wq, ws, r=r), (y + r.float()).to(BF))


def test_extreme_codes():
    """-128 in both operands, sums at the end of int32."""
    for k, code in ((131056, -128), (133136, 127)):
        xq = torch.full((2, k), code, dtype=torch.int8, device="cuda")
        wq = torch.full((8, k), code, dtype=torch.int8, device="cuda")
        wq[1] = -code if code == 127 else 127
        one = lambda n: torch.ones(n, device="cuda")  # noqa: E731
        assert torch.equal(gemm_int8(xq, one(2), wq, one(8)), _want(xq, one(2), wq, one(8)))


@pytest.mark.parametrize("m,k,ns", [(1, 256, (512, 128, 128)), (1, 4096, (4096, 1024, 1024)), (40, 640, (1000, 8, 264)),
                                    (102, 400, (2048, 1024)), (300, 128, (4096, 1024, 1024)), (33, 80, (64, 16, 24)),
                                    (4096, 128, (4096, 64, 64)), (5, 128, (4104,)), (7, 64, (8, 0, 16))])
def test_products_in_one_call_equal_separate_ones(m, k, ns):
    ops = [_operands(m, n, k, n) for n in ns]
    xq, xs = ops[0][:2]
    outs = [torch.full((m, n), 7.0, dtype=BF, device="cuda") for n in ns]
    gemm_int8_multi(xq, xs, [o[2] for o in ops], [o[3] for o in ops], outs)
    for (_, _, wq, ws), out in zip(ops, outs):
        assert torch.equal(out, gemm_int8(xq, xs, wq, ws))


def test_rows_do_not_depend_on_the_others():
    xq, xs, wq, ws = _operands(700, 1024, 1040)
    y = gemm_int8(xq, xs, wq, ws)
    for lo, hi in ((0, 1), (5, 37), (100, 400)):
        assert torch.equal(gemm_int8(xq[lo:hi].contiguous(), xs[lo:hi].contiguous(), wq, ws), y[lo:hi])


def test_output_of_a_view_leaves_the_rest():
    """Rows behind the last one are not touched."""
    xq, xs, wq, ws = _operands(37, 72, 96)
    whole = torch.full((60, 72), 7.0, dtype=BF, device="cuda")
    gemm_int8(xq, xs, wq, ws, out=whole[10:47])
    assert torch.equal(whole[10:47], gemm_int8(xq, xs, wq, ws)) and (whole[:10] == 7).all() and (whole[47:] == 7).all()
    q = torch.full((60, 96), 5, dtype=torch.int8, device="cuda")
    s = torch.full((60,), 5.0, device="cuda")
    x = torch.randn(37, 96, device="cuda").to(BF)
    quantize_rows(x, out=q[10:47], scales=s[10:47])
    assert (q[:10] == 5).all() and (q[47:] == 5).all() and (s[:10] == 5).all() and (s[47:] == 5).all()


def test_layer_as_it_is_used_in_a_graph_and_on_a_stream():
    """Norm, Q/K/V, gate|up, gate, down with the residual: eager, on a stream of its
    own, and captured with other inputs and eager work between the replays."""
    g = torch.Generator(device="cuda").manual_seed(3)
    dm, dff, m = 512, 1408, 37
    gain = (1 + 0.1 * torch.randn(dm, device="cuda", generator=g)).to(BF)
    weights = [quantize_rows(torch.randn(n, k, device="cuda", generator=g) * k ** -0.5)
               for n, k in ((dm, dm), (128, dm), (128, dm), (2 * dff, dm), (dm, dff))]
    x = torch.randn(m, dm, device="cuda", generator=g).to(BF)
    others = [torch.randn(m, dm, device="cuda", generator=g).to(BF) for _ in range(3)]

    def layer(x):
        h, hs = rmsnorm_int8(x, gain, 1e-5)
        qkv = [torch.empty(m, w.shape[0], dtype=BF, device="cuda") for w, _ in weights[:3]]
        gemm_int8_multi(h, hs, [w for w, _ in weights[:3]], [s for _, s in weights[:3]], qkv)
        o = gemm_int8(*quantize_rows(qkv[0]), *weights[0], r=x)
        a = silu_mul_int8(gemm_int8(*rmsnorm_int8(o, gain, 1e-5), *weights[3]))
        return qkv + [gemm_int8(*a, *weights[4], r=o)]
    want = layer(x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = layer(x)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    wants = [layer(t) for t in others]
    held = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer(held)
    for i in (0, 2, 1, 0):
        held.copy_(others[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, wants[i]))
        layer(x)
        torch.cuda.synchronize()
    # against the oracle, from the codes on: the chain's last product
    o = gemm_int8(*quantize_rows(want[0]), *weights[0], r=x)
    aq, as_ = silu_mul_int8(gemm_int8(*rmsnorm_int8(o, gain, 1e-5), *weights[3]))
    ref = Q.product(aq.cpu().numpy(), as_.cpu().numpy(), weights[4][0].cpu().numpy(), weights[4][1].cpu().numpy(), _np(o))
    assert (np.abs(_np(want[3]) - ref) <= 2.0 ** -8 * np.abs(ref) + 1e-5).all()


def test_no_rows_and_no_columns():
    wq, ws = quantize_rows(torch.ones(8, 32, dtype=BF, device="cuda"))
    q, s = quantize_rows(torch.empty(0, 32, dtype=BF, device="cuda"))
    assert q.shape == (0, 32) and s.shape == (0,) and gemm_int8(q, s, wq, ws).shape == (0, 8)
    x = quantize_rows(torch.ones(3, 32, dtype=BF, device="cuda"))
    assert gemm_int8(*x, wq[:0], ws[:0]).shape == (3, 0)
