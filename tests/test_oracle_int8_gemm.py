"""Oracle pins of the int8 projections (readings Q1-Q3), and the refusals of
their entry points and of the binding (host only)."""
import ctypes
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import int8 as Q
from paper_2609_04875_amd import _native as N
from paper_2609_04875_amd import int8


def test_worked_rows():
    codes, s = Q.quantize_rows(np.array([[127.0, -63.5, 62.5, 0.5, 1.5, -0.49], [0, 0, 0, 0, 0, 0],
                                         [1, np.nan, 0, 0, 0, 0], [1, -np.inf, 0, 0, 0, 0]]))
    assert codes[0].tolist() == [127, -64, 62, 0, 2, 0] and s[0] == 1       # ties to even
    assert s[1] == 0 and not codes[1:].any() and np.isnan(s[2:]).all()


def test_error_of_rows_and_products():
    """|code s - y| <= s / 2 (and the quotient's rounding), so a product is off by at
    most sum (|x| ws + |w| xs) / 2 + k xs ws / 4."""
    rng = np.random.default_rng(0)
    x, w = rng.standard_normal((9, 256)).astype(np.float32), rng.standard_normal((16, 256)).astype(np.float32)
    (xq, xs), (wq, ws) = Q.quantize_rows(x), Q.quantize_rows(w)
    assert (np.abs(xq * xs[:, None].astype(np.float64) - x) <= 0.5 * xs[:, None] * (1 + 1e-4)).all()
    y, want = Q.product(xq, xs, wq, ws), x.astype(np.float64) @ w.astype(np.float64).T
    bound = (np.abs(x).sum(1)[:, None] * ws + np.abs(w).sum(1) * xs[:, None]) / 2 + 256 * xs[:, None] * ws / 4
    assert (np.abs(y - want) <= bound * (1 + 1e-4)).all()
    assert np.abs(y - want).mean() < 0.02 * np.abs(want).mean()


def test_largest_k_stays_in_int32():
    assert 127 * 127 * 133136 < 2 ** 31 <= 127 * 127 * (133136 + 16)
    assert 128 * 128 * 131056 < 2 ** 31 <= 128 * 128 * (131056 + 16)


def _p(x):
    return ctypes.c_void_p(x)


@pytest.mark.parametrize("change,code", [
    ({}, N.OK), ({"k": 24}, N.EUNSUPPORTED), ({"k": 133152}, N.EUNSUPPORTED), ({"k": 0}, N.EINVAL), ({"m": -1}, N.EINVAL),
    ({"x": 8, "m": 1}, N.EINVAL), ({"q": 8, "m": 1}, N.EINVAL), ({"s": 2, "m": 1}, N.EINVAL), ({"x": 0, "m": 1}, N.EINVAL),
    ({"q": 0, "m": 1}, N.EINVAL), ({"s": 0, "m": 1}, N.EINVAL)])
def test_rows_are_refused(change, code):
    """Nothing runs: m = 0, or a refusal before any device call."""
    a = {"m": 0, "k": 32, "x": 16, "q": 16, "s": 16, **change}
    L = N.lib
    assert L.pgsr_quantize_rows_int8(a["m"], a["k"], N.BF16, _p(a["x"]), _p(a["q"]), _p(a["s"]), None) == code
    assert L.pgsr_rmsnorm_int8(a["m"], a["k"], _p(a["x"]), _p(16), 1e-5, _p(a["q"]), _p(a["s"]), None) == code
    assert L.pgsr_silu_mul_int8(a["m"], a["k"], _p(a["x"]), _p(a["q"]), _p(a["s"]), None) == code


def test_rows_refuse_types_and_eps():
    L = N.lib
    assert L.pgsr_quantize_rows_int8(0, 32, N.FP8_E4M3, None, None, None, None) == N.EUNSUPPORTED
    for eps in (-1.0, float("nan"), float("inf")):
        assert L.pgsr_rmsnorm_int8(0, 32, None, None, eps, None, None, None) == N.EINVAL
    assert L.pgsr_rmsnorm_int8(1, 32, _p(16), None, 0.0, _p(16), _p(16), None) == N.EINVAL
    assert L.pgsr_rmsnorm_int8(1, 32, _p(16), _p(8), 0.0, _p(16), _p(16), None) == N.EINVAL


@pytest.mark.parametrize("change,code", [
    ({"m": 0}, N.OK), ({"n": 0}, N.OK), ({"n": 12}, N.EUNSUPPORTED), ({"n": -8}, N.EINVAL), ({"k": 8}, N.EUNSUPPORTED),
    ({"k": 133152}, N.EUNSUPPORTED), ({"k": 0}, N.EINVAL), ({"m": -1}, N.EINVAL), ({"x": 8}, N.EINVAL), ({"w": 4}, N.EINVAL),
    ({"ws": 8}, N.EINVAL), ({"xs": 2}, N.EINVAL), ({"y": 4}, N.EINVAL), ({"r": 4}, N.EINVAL), ({"x": 0}, N.EINVAL),
    ({"w": 0}, N.EINVAL), ({"xs": 0}, N.EINVAL), ({"ws": 0}, N.EINVAL), ({"y": 0}, N.EINVAL),
    ({"m": 2 ** 31 - 1, "n": 4096}, N.ERANGE)])
def test_products_are_refused(change, code):
    a = {"m": 4, "n": 16, "k": 32, "x": 16, "xs": 16, "w": 16, "ws": 16, "r": 0, "y": 16, **change}
    assert N.lib.pgsr_gemm_int8(a["m"], a["n"], a["k"], _p(a["x"]), _p(a["xs"]), _p(a["w"]), _p(a["ws"]), _p(a["r"]),
                                _p(a["y"]), None) == code
    if a["r"] == 0:
        two = lambda t, v: (t * 2)(v, v)  # noqa: E731
        ptr = lambda v: two(ctypes.c_void_p, v)  # noqa: E731
        assert N.lib.pgsr_gemm_int8_multi(a["m"], a["k"], 2, two(ctypes.c_int32, a["n"]), _p(a["x"]), _p(a["xs"]),
                                          ptr(a["w"]), ptr(a["ws"]), ptr(a["y"]), None) == code


def test_multi_refuses_its_count_and_arrays():
    n = (ctypes.c_int32 * 4)(8, 8, 8, 8)
    p = (ctypes.c_void_p * 4)(16, 16, 16, 16)
    for count in (0, 4, -1):
        assert N.lib.pgsr_gemm_int8_multi(0, 32, count, n, None, None, p, p, p, None) == N.EINVAL
    assert N.lib.pgsr_gemm_int8_multi(0, 32, 1, None, None, None, p, p, p, None) == N.EINVAL
    assert N.lib.pgsr_gemm_int8_multi(0, 32, 1, n, None, None, p, None, p, None) == N.EINVAL


class OnDevice(torch.Tensor):
    """A host tensor that says it is on the device; nobody follows its pointer here."""
    is_cuda = True
    device = torch.device("cuda", 0)

    def get_device(self):
        return 0


def _new(*shape, dtype=torch.int8):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


@pytest.fixture
def calls(monkeypatch):
    made = []
    names = ("pgsr_gemm_int8", "pgsr_gemm_int8_multi", "pgsr_quantize_rows_int8", "pgsr_rmsnorm_int8", "pgsr_silu_mul_int8")
    monkeypatch.setattr(N, "lib", SimpleNamespace(**{n: (lambda *a, n=n: made.append((n, a)) or 0) for n in names}))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return made


STREAM = SimpleNamespace(cuda_stream=0)
F, B = torch.float32, torch.bfloat16


@pytest.mark.parametrize("change", [
    {}, {"xs": (4,)}, {"ws": (23,)}, {"w": (24, 48)}, {"r": (5, 23)}, {"out": (4, 24)}, {"x_dtype": torch.uint8},
    {"w_dtype": torch.uint8}, {"s_dtype": torch.float64}, {"out_dtype": torch.float16}, {"view": True}, {"device": 1}])
def test_the_binding_checks_a_product(change, calls, monkeypatch):
    x, w = _new(5, 32, dtype=change.get("x_dtype", torch.int8)), _new(*change.get("w", (24, 32)), dtype=change.get("w_dtype", torch.int8))
    if change.get("view"):
        x = _new(5, 64)[:, ::2]
    xs, ws = _new(*change.get("xs", (5,)), dtype=change.get("s_dtype", F)), _new(*change.get("ws", (24,)), dtype=F)
    r, out = _new(*change.get("r", (5, 24)), dtype=B), _new(*change.get("out", (5, 24)), dtype=change.get("out_dtype", B))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: change.get("device", 0))
    run = lambda: int8.gemm_int8(x, xs, w, ws, r=r, out=out, stream=STREAM)  # noqa: E731
    multi = lambda: int8.gemm_int8_multi(x, xs, [w], [ws], [out], stream=STREAM)  # noqa: E731
    if change:
        with pytest.raises(ValueError):
            run()
        if "r" not in change:
            with pytest.raises(ValueError):
                multi()
        assert not calls
    else:
        assert run() is out and multi()[0] is out
        assert calls[0][1][:3] == (5, 24, 32) and calls[0][1][3:9] == tuple(t.data_ptr() for t in (x, xs, w, ws, r, out))
        with pytest.raises(ValueError):
            int8.gemm_int8_multi(x, xs, [w], [ws, ws], [out], stream=STREAM)
        calls.clear()
        int8.gemm_int8_multi(x, xs, [], [], [], stream=STREAM)       # the library refuses the count
        assert calls[0][1][2] == 0


def test_the_binding_checks_rows(calls, monkeypatch):
    x, q, s = _new(5, 32, dtype=B), _new(5, 32), _new(5, dtype=F)
    for bad in (_new(32, dtype=B), _new(5, 32, dtype=torch.float16), _new(5, 64, dtype=B)[:, ::2]):
        with pytest.raises(ValueError):
            int8.quantize_rows(bad, out=q, scales=s, stream=STREAM)
    for kw in ({"out": _new(5, 31), "scales": s}, {"out": q, "scales": _new(4, dtype=F)}, {"out": _new(5, 32, dtype=torch.uint8), "scales": s}):
        with pytest.raises(ValueError):
            int8.quantize_rows(x, stream=STREAM, **kw)
        with pytest.raises(ValueError):
            int8.rmsnorm_int8(x, _new(32, dtype=B), 1e-5, stream=STREAM, **kw)
    with pytest.raises(ValueError):
        int8.rmsnorm_int8(x, _new(31, dtype=B), 1e-5, out=q, scales=s, stream=STREAM)
    with pytest.raises(ValueError):
        int8.rmsnorm_int8(x.float(), _new(32, dtype=B), 1e-5, out=q, scales=s, stream=STREAM)
    with pytest.raises(ValueError):
        int8.silu_mul_int8(_new(5, 63, dtype=B), out=q, scales=s, stream=STREAM)
    assert not calls
    int8.silu_mul_int8(_new(5, 64, dtype=B), out=q, scales=s, stream=STREAM)
    assert calls[0][0] == "pgsr_silu_mul_int8" and calls[0][1][:2] == (5, 32)
