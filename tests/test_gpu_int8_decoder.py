"""Decoder layers with int8 projections and an int8 cache (reading Q4): replay
from a crop inside a block equals the full reset bit for bit (Theorem 1) and
the calls it is made of, is near the fp64 oracle and the bf16 layers, and captured
replays equal eager ones."""
import numpy as np
import pytest
import torch

from gpu_helpers import log
from oracle import bf16_round
from oracle import int8 as Q

from paper_2609_04875_amd import (BF16, F32, FP8_E4M3, INT8, DecoderReplay, KVPool, gemm_int8, quantize_rows,
                                  quantize_weights, rmsnorm_int8, rope_, silu_mul_int8, workspace_bytes)

pytestmark = pytest.mark.gpu

EPS, THETA = 1e-5, 5e5


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(torch.bfloat16)


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def _weights(rng, n_layers, dm, hq, hkv, d, dff):
    shapes = {"wq": (hq * d, dm), "wk": (hkv * d, dm), "wv": (hkv * d, dm), "wo": (dm, hq * d),
              "w_gate_up": (2 * dff, dm), "w_down": (dm, dff)}
    return [{**{name: _dev(rng.standard_normal(s) * s[1] ** -0.5) for name, s in shapes.items()},
             **{g: _dev(1 + 0.1 * rng.standard_normal(dm)) for g in ("g_attn", "g_mlp")}} for _ in range(n_layers)]


def _setup(hq, hkv, d, kv, seed, T=300, P=203, Tc=330, dff=384, ws=0):
    rng = np.random.default_rng(seed)
    dm = hq * d
    w = _weights(rng, 2, dm, hq, hkv, d, dff)
    x = bf16_round(rng.standard_normal((T, dm)))
    xc = np.concatenate([x[:P], bf16_round(3 * rng.standard_normal((Tc - P, dm)))])
    mk = lambda weights, kv_dtype: DecoderReplay(weights, hq, hkv, d, EPS, THETA, n_blocks=3 * (-(-Tc // 16)) + 8,  # noqa: E731
                                                 max_seqs=2, max_blocks_per_seq=32, workspace_bytes=ws, kv_dtype=kv_dtype)
    return w, quantize_weights(w), x, xc, mk


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (7, 1, 64), (4, 1, 128)])
@pytest.mark.parametrize("kv", [INT8, BF16])
def test_int8_decoder_matches_oracle_and_full_reset(hq, hkv, d, kv):
    log(f"int8 decoder layers {hq}/{hkv}/{d} cache {kv}")
    T, P = 300, 203
    w, w8, x, xc, mk = _setup(hq, hkv, d, kv, hq)
    dec = mk(w8, kv)
    dec.replay(0, _dev(xc))
    assert dec.crop([0], [P]) == 0
    out = dec.replay(0, _dev(x[P:]))
    full = dec.full_reset(1, _dev(x))
    torch.cuda.synchronize()
    assert torch.equal(full[P:], out)                                 # Theorem 1, bitwise
    host = [{**{n: tuple(t.cpu().numpy() for t in w8[i][n]) for n in ("wq", "wk", "wv", "wo", "w_gate_up", "w_down")},
             **{g: _f64(w8[i][g]) for g in ("g_attn", "g_mlp")}} for i in range(2)]
    ref = Q.decoder_layers(x, host, hq, hkv, d, EPS, THETA, kv == INT8)[P:]
    # fp32 here and fp64 there (and P in bf16) move a value by far less than a step of
    # the codes it is rounded to, so a code is off by one at most: 1/127 of its row's
    # largest value, four and a half standard deviations, or 3.5% of a typical value if
    # every code moved.  A branch has two such places in a row (the norm's rows and the
    # attention's, or the gate's: 5%, and 3.5% of the gate's factors once more: 6%), the
    # two layers four branches, whose errors add as squares: 12% of x, where a wrong
    # step, order or scale is off by all of it.
    off = lambda a, b: np.sqrt(np.square(a - b).sum() / np.square(b).sum())  # noqa: E731
    log(f"off the oracle by {off(_f64(out), ref):.2e}")
    assert off(_f64(out), ref) <= 0.12
    # the bf16 layers: codes round by 1/sqrt(12) of a step, 1% of a typical value, in both
    # operands of a product; two products in a row and four branches: 1.4% * 2 * sqrt(2)
    plain = _f64(mk(w, BF16).full_reset(0, _dev(x))[P:])
    log(f"off the bf16 layers by {off(_f64(out), plain):.2e}")
    assert off(_f64(out), plain) <= 0.04


def test_wide_int8_layers_equal_the_full_reset():
    """States of 4096 values: a suffix of 1 to 300 tokens takes other kernels of the
    norm and the products than the whole session does, with the same bits."""
    hq, hkv, d = 32, 8, 128
    log("int8 decoder layer of 4096")
    w, x, xc = _setup(hq, hkv, d, INT8, 5, T=700, P=1, Tc=720, dff=4112)[1:4]
    mk = lambda: DecoderReplay(w[:1], hq, hkv, d, EPS, THETA, n_blocks=48, max_seqs=1, max_blocks_per_seq=48,  # noqa: E731
                               kv_dtype=INT8)
    full = mk().full_reset(0, _dev(x))
    for S in (1, 40, 300):
        dec = mk()
        dec.replay(0, _dev(np.concatenate([x[:700 - S], xc[700 - S:]])))
        assert dec.crop([0], [700 - S]) == 0
        assert torch.equal(dec.replay(0, _dev(x[700 - S:])), full[700 - S:]), S


@pytest.mark.parametrize("kv", [INT8, BF16])
def test_int8_decoder_is_the_calls_it_is_made_of(kv):
    """The layers, written out in the public calls: the same bits."""
    hq, hkv, d, T = 4, 2, 64, 77
    _, w8, x, _, mk = _setup(hq, hkv, d, kv, 12)
    pool = KVPool(2, hq, hkv, d, 32, 1, 32, kv)
    t, n = _dev(x[:T]), T
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    new = lambda *shape: torch.empty(*shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    for li, w in enumerate(w8):
        q, k, v, o = new(n, hq, d), new(n, hkv, d), new(n, hkv, d), new(n, hq * d)
        h = rmsnorm_int8(t, w["g_attn"], EPS)
        for name, y in (("wq", q), ("wk", k), ("wv", v)):
            gemm_int8(*h, *w[name], out=y)
        rope_(q, pos, THETA)
        rope_(k, pos, THETA)
        assert pool.replay(li, [0], [n], q, k, v, o, d ** -0.5, commit=li == 1) == 0
        t = gemm_int8(*quantize_rows(o), *w["wo"], r=t)
        t = gemm_int8(*silu_mul_int8(gemm_int8(*rmsnorm_int8(t, w["g_mlp"], EPS), *w["w_gate_up"])), *w["w_down"], r=t)
    assert torch.equal(mk(w8, kv).replay(0, _dev(x[:T])), t)


def test_captured_int8_restore_replay_matches_eager():
    log("int8 decoder restore + replay as a HIP graph")
    T, P = 300, 203
    w, w8, x, xc, mk = _setup(4, 2, 64, INT8, 99)
    dec = mk(w8, INT8)
    dec.replay(0, _dev(xc))
    torch.cuda.synchronize()
    saved = dec.pool.save_meta()
    assert dec.crop([0], [P]) == 0
    want = dec.replay(0, _dev(x[P:])).clone()
    torch.cuda.synchronize()
    after = dec.pool.save_meta()
    dec.pool.load_meta(saved)
    cap = dec.capture_restore_replay(0, P, _dev(x[P:]))
    for i in range(3):
        dec.pool.load_meta(saved)
        got = cap.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want), f"graph replay {i} differs from the eager replay"
        assert all(torch.equal(a, b) for a, b in zip(dec.pool.save_meta(), after)), f"replay {i} tables"
        dec.pool.refresh()
        full = dec.full_reset(1, _dev(x))
        torch.cuda.synchronize()
        assert torch.equal(full[P:], want)
        assert dec.crop([1], [0]) == 0
        torch.cuda.synchronize()


def test_single_tokens_through_an_int8_decoder():
    """Re-decode, a token at a time on the decode kernel: near the replay of all of
    them at once (other rounding orders)."""
    hq, hkv, d = 4, 2, 64
    w, w8, x, xc, mk = _setup(hq, hkv, d, INT8, 5, ws=workspace_bytes(hq, d, 8, 8))
    a, b = mk(w8, INT8), mk(w8, INT8)
    a.replay(0, _dev(x[:290]))
    b.replay(0, _dev(x[:290]))
    one = torch.cat([a.replay(0, _dev(x[t:t + 1])) for t in range(290, 300)])
    at_once = b.replay(0, _dev(x[290:]))
    # codes off by one where the attention rounds in another order, as above
    one, at_once = _f64(one), _f64(at_once)
    assert np.square(one - at_once).sum() <= 0.12 ** 2 * np.square(at_once).sum()


def test_fp8_cache_and_refusals():
    w, w8, x, _, mk = _setup(4, 2, 64, INT8, 6)
    dec = mk(w, FP8_E4M3)
    dec.pool.set_kv_scales([0.02] * 2, [0.02] * 2)
    out, want = _f64(dec.full_reset(0, _dev(x))), _f64(mk(w, BF16).full_reset(0, _dev(x)))
    # codes of four significant bits: half a step is at most 2^-4 of a value of K and V;
    # each of two layers' attention takes both
    assert np.square(out - want).sum() <= (4 * 2.0 ** -4) ** 2 * np.square(want).sum()
    with pytest.raises(ValueError):
        mk([w[0], w8[1]], INT8)                                    # one layer of each
    with pytest.raises(ValueError):
        mk([{**w8[0], "wo": w[0]["wo"]}], INT8)
    with pytest.raises(ValueError):
        mk(w8, F32)
