"""Oracle pins of the int8 KV cache (readings I1, I2): worked rows, the error
bound, and that a row's stored form depends on its own values alone.  Host-side
refusals of the exponents' entry point."""
import ctypes

import numpy as np
import pytest

import oracle
from oracle import bf16_round, int8_read, int8_row


def test_worked_rows():
    # a = 1: floor(log2 1) - 6 = -6, steps of 1/64
    codes, e = int8_row(np.array([1.0, -0.5, 1 / 64, 1 / 128, 3 / 128, -1 / 128]))
    assert e == -6 and codes.tolist() == [64, -32, 1, 0, 2, 0]          # ties to even
    # 1.9921875 = 127.5 / 64 rounds to 128, past the largest code
    codes, e = int8_row(np.array([1.9921875, -1.9921875, 1.984375]))
    assert e == -6 and codes.tolist() == [127, -127, 127]
    codes, e = int8_row(np.zeros(4))
    assert e == -100 and not codes.any()
    codes, e = int8_row(np.array([np.inf, 1.0, -np.inf, 2.0 ** 106]))
    assert e == 100 and codes.tolist() == [127, 0, -127, 64]
    codes, e = int8_row(np.array([2.0 ** -101, 2.0 ** -102, 2.0 ** -100, np.nan]))
    assert e == -100 and codes.tolist() == [0, 0, 1, 0]


def test_error_is_half_a_step_of_the_largest_value():
    rng = np.random.default_rng(0)
    x = bf16_round(rng.standard_normal((500, 64)) * np.exp(3 * rng.standard_normal((500, 1))))
    codes, e = int8_row(x)
    top = np.abs(codes).max(-1)
    assert ((top >= 64) & (top <= 127)).all()
    assert (np.abs(int8_read(x) - x) <= np.ldexp(0.5, e)[:, None]).all()
    assert (np.ldexp(0.5, e) <= np.abs(x).max(-1) / 128).all()


def test_read_back_values_are_bf16_and_stay():
    rng = np.random.default_rng(1)
    x = bf16_round(rng.standard_normal((200, 128)) * 7)
    once = int8_read(x)
    assert np.array_equal(bf16_round(once), once) and np.array_equal(int8_read(once), once)


def test_rows_do_not_depend_on_their_neighbours():
    """What lets a crop keep any number of tokens: the kept rows' stored form is
    that of a pool that never saw the others."""
    rng = np.random.default_rng(2)
    x = bf16_round(rng.standard_normal((40, 2, 64)))
    loud = np.concatenate([x[:21], 1e6 * x[21:]])
    a, b = int8_row(x)[0], int8_row(loud)[0]
    assert np.array_equal(a[:21], b[:21])
    pool = oracle.PoolModel(8, 1, 8, 16, n_layers=1, n_kv_heads=2, head_dim=64, kv_int8=True)
    q = np.zeros((40, 2, 64))
    oracle.prefill(pool, 0, [0], [40], q, loud, loud, 1.0)
    assert pool.crop([0], [21]) == 0
    assert np.array_equal(pool.gather(0, 0, 21)[0], int8_read(x[:21]))


def test_nan_token_reads_as_nan_key():
    pool = oracle.PoolModel(2, 1, 2, 16, n_layers=1, n_kv_heads=2, head_dim=64, kv_int8=True)
    k, v = np.ones((3, 2, 64)), np.ones((3, 2, 64))
    k[1, 0, 5] = np.nan
    v[2, 1, 7] = np.nan
    assert pool.reserve([0], [3]) == 0
    pool.write(0, 0, 0, k, v)
    gk, gv = pool.gather(0, 0, 3)
    assert np.isnan(gk[1, 0]).all() and np.isnan(gk[2, 1]).all() and np.isfinite(gv).all()
    assert np.isfinite(gk[0]).all() and np.isfinite(gk[1, 1]).all() and gv[2, 1, 7] == 0


def test_exponents_are_refused_without_a_pool():
    from paper_2609_04875_amd import _native as N
    assert N.lib.pgsr_pool_set_kv_exponents(None, ctypes.c_void_p(16)) == N.EINVAL
    out = ctypes.c_void_p()
    fake = ctypes.c_void_p(16)   # never dereferenced: validation fails first
    for bad, code in (({"hq": 33, "hkv": 1}, N.EUNSUPPORTED), ({"d": 96}, N.EUNSUPPORTED), ({"B": 8}, N.EUNSUPPORTED),
                      ({"hq": 30}, N.EUNSUPPORTED), ({"nb": 0}, N.EINVAL)):
        a = {"hq": 32, "hkv": 8, "d": 128, "B": 16, "nb": 64, **bad}
        assert N.lib.pgsr_pool_create(1, a["hq"], a["hkv"], a["d"], a["B"], N.INT8, a["nb"], 2, 8, fake, fake, fake,
                                      fake, fake, fake, fake, None, 0, None, None, ctypes.byref(out)) == code


def test_lists_of_a_call_convert_as_ints(monkeypatch):
    """Sequence ids and lengths of any integer-like type, and a length past 32 bits,
    which must not pass for the one its low bits name."""
    import types

    import torch
    from paper_2609_04875_amd import _native as N, pool as P
    for values in ([3, 1], (3, 1), b"\x03\x01", np.array([3, 1]), np.array([3, 1], np.int32), torch.tensor([3, 1]),
                   [3.0, 1.0], [np.int64(3), True], range(3, 0, -2), N.int32s([3, 1])):
        assert list(N.int32_array(values)) == [3, 1], values
    assert list(N.int32_array([])) == [0]
    seen = []
    pool = types.SimpleNamespace(_h=None, dtype=torch.bfloat16, _dev=0, hq=8, hkv=2, d=64,
                                 recomputed_tokens=ctypes.c_int64(0))
    monkeypatch.setattr(P, "_dev_ptr", lambda t, dt, name, dv, numel: seen.append((name, numel)))
    monkeypatch.setattr(P, "_stream_ptr", lambda stream, dv=None: None)
    P.KVPool._prefill(pool, lambda *a: 0, 0, [0], [2 ** 32 + 3], None, None, None, None, 1.0, True, None)
    assert seen[0] == ("q", (2 ** 32 + 3) * 8 * 64) and seen[1] == ("k", (2 ** 32 + 3) * 2 * 64)
    with pytest.raises(ValueError):
        P.KVPool._prefill(pool, lambda *a: 0, 0, [0, 1], [1, -2 ** 40], None, None, None, None, 1.0, True, None)
