"""Int8 KV cache (readings I1, I2): the append stores the oracle's codes and
exponents bit for bit; attention over them equals, bit for bit, a bf16 pool that
holds the values read back (every code times its power of two is a bf16 value)
wherever the two run the same arithmetic, and matches the fp64 oracle on those
values in decode steps; crops to any token, forks and batching leave no trace
(selective replay = full reset); a NaN reaches the rows that see it and no others."""
import numpy as np
import pytest
import torch

import oracle
import workloads as W
from gpu_helpers import dev, log, storage_f64

pytestmark = pytest.mark.gpu


def _blocks(n, B=16):
    return -(-n // B)


def _pool(geom, n_blocks, max_seqs, max_bps, B=16, n_layers=1, split_q=0, max_splits=16, dtype="int8"):
    from paper_2609_04875_amd import BF16, INT8, KVPool, workspace_bytes
    ws = workspace_bytes(geom.n_q_heads, geom.head_dim, split_q, max_splits) if split_q else 0
    return KVPool(n_layers, geom.n_q_heads, geom.n_kv_heads, geom.head_dim, n_blocks, max_seqs, max_bps,
                  INT8 if dtype == "int8" else BF16, B, workspace_bytes=ws)


def _stored(pool, layer, seq, n):
    """Codes [n, Hkv, d] and exponent bytes [n, Hkv] of logical tokens 0..n-1 (K, V)."""
    torch.cuda.synchronize()
    tables = pool.block_tables[seq].long()
    pos = torch.arange(n, device="cuda")
    blk, slot = tables[pos // pool.B], pos % pool.B
    ex = pool.kv_exponents[layer][blk, :, :, slot]
    return tuple(t.cpu().numpy().astype(np.int64) for t in (
        pool.k_cache[layer][blk, :, slot, :], pool.v_cache[layer][blk, :, :, slot], ex[..., 0], ex[..., 1]))


def _read(pool, layer, seq, n):
    ck, cv, ek, ev = _stored(pool, layer, seq, n)
    k = np.ldexp(ck.astype(np.float64), (ek - 127)[..., None])
    return np.where((ek == 255)[..., None], np.nan, k), np.ldexp(cv.astype(np.float64), (ev - 127)[..., None])


def _bf16(x):
    return dev(W.f32_to_bf16_bits(np.asarray(x, np.float32)), "bf16")


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def _rand(rng, *shape):
    """bf16 values whose rows differ in size, with a few large channels."""
    x = rng.standard_normal(shape) * np.exp(0.5 * rng.standard_normal(shape[:-1] + (1,)))
    return oracle.bf16_round(x * np.exp(0.7 * rng.standard_normal(shape[-1])))


def _decode_bound(q, k, v, pos0, scale, want):
    """The decode kernel multiplies unrounded scores; its weights are rounded to
    bf16 (half a step: 2^-8 of each) and normalised by the sum of the rounded
    ones, the result is rounded once: 2^-8 (sum p |v| + |o|) + 2^-8 |o|, and 1e-5
    of sum p |v| for fp32 exponentials and sums over thousands of keys."""
    mag = oracle.attention(q, k, np.abs(v), pos0, scale)
    return 2.0 ** -8 * (mag + 2 * np.abs(want)) * 1.01 + 1e-5 * mag + 1e-30


def _query_rounding(q, k, v, scale, o):
    """The prefill kernels round a query times the scale to bf16, half a step: 2^-8 of
    each of its values, so a score moves by d_j <= 2^-8 scale sum |q_i k_ij|, a weight
    by a factor within e^(+-2 max d) of its own, and the result by at most
    e^(2 max d) sum p_j d_j (|v_j| + |o|)."""
    group, out = q.shape[0] // k.shape[1], np.zeros_like(o)
    for h in range(q.shape[0]):
        kh, vh = k[:, h // group], v[:, h // group]
        s = kh @ q[h] * scale
        p = np.exp(s - s.max())
        d = 2.0 ** -8 * scale * (np.abs(kh) @ np.abs(q[h]))
        w = p / p.sum() * d
        out[h] = np.exp(2 * d.max()) * (w @ np.abs(vh) + w.sum() * np.abs(o[h]))
    return out


def _special_rows(x, at):
    """Rows that saturate, vanish, tie, hold zeros, infinities and subnormals."""
    x[at + 0, 0] = 0.0
    x[at + 1, 0] *= 2.0 ** 110
    x[at + 2, 0, :4] = [np.inf, -np.inf, 1.0, -2.0 ** 106]
    x[at + 3, 0] = 2.0 ** -133                                    # the smallest bf16 subnormal
    x[at + 4, 0, :6] = [1.9921875, -1.9921875, 1.0078125, 0.0234375, -0.0, 0.0078125]
    x[at + 5, 0] *= 2.0 ** -100
    return x


@pytest.mark.parametrize("hq,hkv,d,B", [(8, 2, 64, 16), (28, 4, 128, 32), (5, 5, 128, 64)])
def test_append_is_bit_exact(hq, hkv, d, B):
    """Two layers, two sequences, two appends (the second into a partial block)."""
    log(f"int8 append {hq}/{hkv}/{d} B={B}")
    geom = W.AttnGeometry(hq, hkv, d)
    rng = np.random.default_rng(hq)
    pool = _pool(geom, 24, 2, 8, B, n_layers=2)
    have = {s: {l: ([], []) for l in (0, 1)} for s in (0, 1)}
    for sizes in [(37, 19), (12, 40)]:
        S = sum(sizes)
        q = torch.zeros((S, hq, d), dtype=torch.bfloat16, device="cuda")
        for layer in (0, 1):
            k, v = _special_rows(_rand(rng, S, hkv, d), 3), _special_rows(_rand(rng, S, hkv, d), 7)
            k, v = (storage_f64(W.f32_to_bf16_bits(x.astype(np.float32)), "bf16") for x in (k, v))
            k[14, 1 % hkv, 3] = v[15, 0, 9] = np.nan
            assert pool.replay(layer, [0, 1], sizes, q, _bf16(k), _bf16(v), torch.empty_like(q), 0.1,
                               commit=layer == 1) == 0
            off = 0
            for s, n in zip((0, 1), sizes):
                have[s][layer][0].append(k[off:off + n])
                have[s][layer][1].append(v[off:off + n])
                off += n
    for s in (0, 1):
        for layer in (0, 1):
            k, v = (np.concatenate(x) for x in have[s][layer])
            ck, cv, ek, ev = _stored(pool, layer, s, len(k))
            wk, we = oracle.int8_row(k)
            xk, xe = oracle.int8_row(v)
            nan = (np.isnan(k) | np.isnan(v)).any(-1)
            assert np.array_equal(ck, np.where(nan[..., None], 0, wk))
            assert np.array_equal(ek, np.where(nan, 255, we + 127))
            assert np.array_equal(cv, xk) and np.array_equal(ev, xe + 127)


def test_append_off_the_16_byte_boundary():
    geom = W.AttnGeometry(4, 2, 64)
    rng = np.random.default_rng(5)
    a, b = _pool(geom, 8, 1, 8), _pool(geom, 8, 1, 8)
    k, v, q = (_bf16(_rand(rng, 41, h, 64)) for h in (2, 2, 4))

    def shifted(x):
        return torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(x.shape).copy_(x)
    assert a.replay(0, [0], [41], q, k, v, torch.empty_like(q), 0.1) == 0
    assert b.replay(0, [0], [41], q, shifted(k), shifted(v), torch.empty_like(q), 0.1) == 0
    for x, y in zip(_stored(a, 0, 0, 41), _stored(b, 0, 0, 41)):
        assert np.array_equal(x, y)


@pytest.mark.parametrize("hq,hkv,d,B", [(8, 2, 64, 16), (28, 4, 128, 32), (5, 5, 128, 64), (32, 1, 64, 64), (4, 4, 128, 16)])
def test_single_tokens_store_what_an_append_stores(hq, hkv, d, B):
    """Steps of one token a sequence in a pool with a workspace (the decode kernel
    appends) and without (an append launch): tables, lengths, counts, free stack, codes
    and exponents are the same, whatever the rows hold; committed or not, two layers,
    more sequences than a launch, new blocks and empty sequences among them."""
    log(f"int8 single tokens {hq}/{hkv}/{d} B={B}")
    geom = W.AttnGeometry(hq, hkv, d)
    rng = np.random.default_rng(hq + B)
    n, ctx = 70, [int(x) for x in np.r_[0, 0, B - 1, B, 2 * B, 31, 32, 33, 63, 64, rng.integers(0, 150, 60)]]
    seqs = [int(x) for x in rng.permutation(n)]
    blocks = sum(_blocks(c + 5, B) for c in ctx)
    pools = [_pool(geom, blocks, n, _blocks(160, B), B, n_layers=2, split_q=n, max_splits=4),
             _pool(geom, blocks, n, _blocks(160, B), B, n_layers=2)]
    for layer in (0, 1):
        x = [_bf16(_rand(rng, sum(ctx), h, d)) for h in (hq, hkv, hkv)]
        for pool in pools:
            assert pool.replay(layer, seqs, ctx, *x, torch.empty_like(x[0]), 0.09, commit=layer == 1) == 0
    for step in range(5):
        for layer in (0, 1):
            q, k, v = (_rand(rng, n, h, d) for h in (hq, hkv, hkv))
            k, v = _special_rows(k, 3), _special_rows(v, 6)
            k[20, hkv - 1, d - 1] = v[21, 0, 9] = np.nan
            x = [_bf16(t) for t in (q, k, v)]
            for pool in pools:
                assert pool.replay(layer, seqs, [1] * n, *x, torch.empty_like(x[0]), 0.09,
                                   commit=layer == 1 and step != 2) == 0
        torch.cuda.synchronize()
        a, b = pools
        top = int(a.free_top)
        assert top == int(b.free_top) and torch.equal(a.free_list[:top], b.free_list[:top])
        assert torch.equal(a.seq_lens, b.seq_lens) and torch.equal(a.ref_counts, b.ref_counts)
        for s, c in zip(seqs, ctx):
            m = c + step + (step < 2) + (step == 2)              # step 2 is written over by step 3
            held = _blocks(m, B)
            assert torch.equal(a.block_tables[s, :held], b.block_tables[s, :held])
            for layer in (0, 1):
                for y, z in zip(_stored(a, layer, s, m), _stored(b, layer, s, m)):
                    assert np.array_equal(y, z), (step, s, layer)


# geometry, block size, kept prefixes, suffixes, contaminated lengths
PREFILL = [
    (W.AttnGeometry(32, 8, 128), 16, (260, 0, 1000), (301, 77, 129), (600, 50, 1100)),
    (W.AttnGeometry(28, 4, 128), 32, (97, 513), (200, 64), (300, 520)),
    (W.AttnGeometry(16, 4, 64), 64, (33, 130), (250, 7), (40, 200)),
    (W.AttnGeometry(4, 4, 128), 64, (5, 700, 64, 63), (1, 900, 65, 2), (5, 701, 70, 64)),
    (W.AttnGeometry(32, 1, 64), 16, (300,), (45,), (320,)),
    (W.AttnGeometry(8, 8, 64), 32, tuple(range(40)), tuple(range(2, 42)), tuple(range(3, 43))),
    (W.AttnGeometry(64, 8, 128), 16, (2100,), (1500,), (2101,)),
]


def _run(pool, data, prefixes, suffixes, contaminated, scale, poison=False):
    """Contaminated prefill, crop, sanitized replay; the replay's output."""
    q, k, v, cq, ck, cv = data
    seqs = list(range(len(prefixes)))
    assert pool.replay(0, seqs, contaminated, cq, ck, cv, torch.empty_like(cq), scale) == 0
    assert pool.crop(seqs, prefixes, poison=poison) == 0
    o = torch.full_like(q, float("nan"))
    assert pool.replay(0, seqs, suffixes, q, k, v, o, scale) == 0
    torch.cuda.synchronize()
    return o


def _episodes(rng, geom, prefixes, suffixes, contaminated, quantised):
    """Packed device inputs of the two runs; ``quantised`` gives what an int8 pool reads."""
    hq, hkv, d = geom.n_q_heads, geom.n_kv_heads, geom.head_dim
    full = [tuple(_rand(rng, P + S, h, d) for h in (hq, hkv, hkv)) for P, S in zip(prefixes, suffixes)]
    extra = [tuple(_rand(rng, C - P, h, d) * (1, 30, 30)[i] for i, h in enumerate((hq, hkv, hkv)))
             for C, P in zip(contaminated, prefixes)]
    f = oracle.int8_read if quantised else (lambda x: x)
    g = [lambda x: x, f, f]
    suffix = [_bf16(g[i](np.concatenate([x[i][P:] for x, P in zip(full, prefixes)]))) for i in range(3)]
    before = [_bf16(g[i](np.concatenate([np.concatenate([x[i][:P], y[i]]) for x, y, P in zip(full, extra, prefixes)])))
              for i in range(3)]
    return suffix + before, full


@pytest.mark.parametrize("case", range(len(PREFILL)))
@pytest.mark.parametrize("kernel", ["auto", "pipelined", "four_wave"])
def test_prefill_equals_a_bf16_pool_of_the_values_read_back(case, kernel):
    """Crop inside a block after a louder contaminated run (poisoned slots), then
    the replay: the bits of the four-wave bf16 kernel on the values read back, and
    the oracle on a sample of rows."""
    geom, B, P, S, C = PREFILL[case]
    log(f"int8 prefill case {case} {kernel}")
    nb = sum(_blocks(max(c, p + s), B) + 1 for p, s, c in zip(P, S, C))
    bps = max(_blocks(max(c, p + s), B) for p, s, c in zip(P, S, C)) + 1
    scale = geom.head_dim ** -0.5
    data, full = _episodes(np.random.default_rng(case), geom, P, S, C, False)
    read, _ = _episodes(np.random.default_rng(case), geom, P, S, C, True)
    pool, ref = (_pool(geom, nb, len(P), bps, B, dtype=t) for t in ("int8", "bf16"))
    pool.set_prefill_kernel(kernel)
    ref.set_prefill_kernel("four_wave")
    o = _run(pool, data, P, S, C, scale, poison=True)
    want = _run(ref, read, P, S, C, scale, poison=True)
    assert torch.equal(o, want)
    off = 0
    for i, (p, s) in enumerate(zip(P, S)):
        k, v = (oracle.int8_read(x) for x in full[i][1:])
        gk, gv = _read(pool, 0, i, p + s)
        assert np.array_equal(gk, k) and np.array_equal(gv, v)
        if i < 2:
            rows = np.unique(np.linspace(0, s * geom.n_q_heads - 1, 60).astype(np.int64))
            ref_rows = oracle.attention(full[i][0][p:], k, v, p, scale, rows=rows)
            got = _f64(o[off:off + s]).reshape(-1, geom.head_dim)[rows]
            d = np.abs(got - ref_rows)
            assert d.sum() <= 1e-2 * np.abs(ref_rows).sum(), (i, d.max())
        off += s


def test_selective_equals_full_reset_bitwise():
    """Theorem 1 with every kept token inside a block that held louder forgotten ones."""
    geom, B, P, S, C = PREFILL[0]
    log("int8 selective vs full reset")
    data, full = _episodes(np.random.default_rng(50), geom, P, S, C, False)
    pool = _pool(geom, sum(_blocks(max(c, p + s)) + 1 for p, s, c in zip(P, S, C)), 3, 80)
    o = _run(pool, data, P, S, C, 0.09)
    fresh = _pool(geom, sum(_blocks(p + s) for p, s in zip(P, S)), 3, 80)
    fq, fk, fv = (_bf16(np.concatenate([x[i] for x in full])) for i in range(3))
    fo = torch.empty_like(fq)
    assert fresh.full_reset(0, [0, 1, 2], [p + s for p, s in zip(P, S)], fq, fk, fv, fo, 0.09) == 0
    at, off = 0, 0
    for p, s in zip(P, S):
        assert torch.equal(fo[off + p:off + p + s], o[at:at + s])
        at, off = at + s, off + p + s
    # restore + replay in one call, on top of the state that is there
    seqs, q = [0, 1, 2], data[0]
    again = torch.empty_like(q)
    assert pool.restore_replay(0, seqs, P, S, q, data[1], data[2], again, 0.09) == 0
    assert torch.equal(again, o) and [pool.seq_len(i) for i in seqs] == [p + s for p, s in zip(P, S)]


DECODE = [   # geometry, block size, cached lengths, new tokens
    (W.AttnGeometry(32, 8, 128), 16, (0, 1, 15, 16, 17, 31, 1330, 5000), (1,) * 8),
    (W.AttnGeometry(28, 4, 128), 32, (3, 700, 64), (4, 1, 3)),
    (W.AttnGeometry(4, 4, 64), 64, (200, 0, 63), (32, 31, 1)),
    (W.AttnGeometry(32, 1, 128), 64, (4097, 130), (1, 1)),
    (W.AttnGeometry(8, 4, 64), 16, tuple(range(70)), (1,) * 70),
]


@pytest.mark.parametrize("case", range(len(DECODE)))
@pytest.mark.parametrize("split", [True, False])
def test_decode_matches_the_oracle(case, split):
    """Single tokens (and a few) against caches from empty on; poisoned slots behind."""
    geom, B, ctx, new = DECODE[case]
    log(f"int8 decode case {case} split={split}")
    hq, hkv, d = geom.n_q_heads, geom.n_kv_heads, geom.head_dim
    rng = np.random.default_rng(300 + case)
    n, scale = len(ctx), d ** -0.5
    # one split: a workspace of a byte takes the decode kernel and holds no partials
    pool = _pool(geom, sum(_blocks(c + s + 3, B) for c, s in zip(ctx, new)), n,
                 max(_blocks(c + s + 3, B) for c, s in zip(ctx, new)), B, split_q=sum(new) if split else 0, max_splits=32)
    if not split:
        from paper_2609_04875_amd import INT8, KVPool
        pool = KVPool(1, hq, hkv, d, pool.n_blocks, n, pool.max_bps, INT8, B, workspace_bytes=16)
    full = [tuple(_rand(rng, c + s + 3, h, d) for h in (hq, hkv, hkv)) for c, s in zip(ctx, new)]
    seqs = list(range(n))
    cat = lambda i, lo, hi: _bf16(np.concatenate([x[i][a:b] for x, a, b in zip(full, lo, hi)]))  # noqa: E731
    ends = [c + s + 3 for c, s in zip(ctx, new)]
    q, k, v = (cat(i, [0] * n, ends) for i in range(3))
    assert pool.replay(0, seqs, ends, q, k, v, torch.empty_like(q), scale) == 0
    assert pool.crop(seqs, ctx, poison=True) == 0
    q, k, v = (cat(i, ctx, [c + s for c, s in zip(ctx, new)]) for i in range(3))
    o = torch.full_like(q, float("nan"))
    assert pool.replay(0, seqs, new, q, k, v, o, scale, commit=False) == 0
    torch.cuda.synchronize()
    off = 0
    for i, (c, s) in enumerate(zip(ctx, new)):
        kk, vv = (oracle.int8_read(x[:c + s]) for x in full[i][1:])
        want = oracle.attention(full[i][0][c:c + s], kk, vv, c, scale)
        bound = _decode_bound(full[i][0][c:c + s], kk, vv, c, scale, want)
        diff = np.abs(_f64(o[off:off + s]) - want)
        assert (diff <= bound).all(), (i, (diff / bound).max())
        off += s
    again = torch.empty_like(o)                                     # uncommitted: the same call again
    assert pool.replay(0, seqs, new, q, k, v, again, scale, commit=False) == 0
    assert torch.equal(o, again)


def test_nan_reaches_the_rows_that_see_it():
    """A NaN in a new token's K or V of one head, prefill and decode kernels: rows
    from that token on, of that head's group, are NaN; the others as without it."""
    geom = W.AttnGeometry(8, 2, 128)
    rng = np.random.default_rng(9)
    for n_new, at, split_q, which in [(150, 70, 0, 1), (150, 70, 0, 2), (8, 3, 8, 1), (8, 3, 8, 2), (8, 0, 8, 2)]:
        log(f"int8 NaN {n_new} {at} {split_q} {which}")
        x = [_rand(rng, 93 + n_new, h, 128) for h in (8, 2, 2)]
        outs = []
        for bad in (False, True):
            pool = _pool(geom, 32, 1, 32, split_q=split_q)
            z = [_bf16(t[:93]) for t in x]
            assert pool.replay(0, [0], [93], *z, torch.empty_like(z[0]), 0.09) == 0
            new = [t[93:].copy() for t in x]
            if bad:
                new[which][at, 1, 17] = np.nan
            new = [_bf16(t) for t in new]
            o = torch.empty_like(new[0])
            assert pool.replay(0, [0], [n_new], *new, o, 0.09) == 0
            outs.append(o)
        clean, got = outs
        assert torch.isnan(got[at:, 4:]).all()
        assert torch.equal(got[:at], clean[:at]) and torch.equal(got[:, :4], clean[:, :4])


def test_rows_of_very_different_size():
    """V rows from 2^-60 to 2^60 and zeros: what the weights carry into the PV
    product keeps its precision; the values are sums in which one scale dominates."""
    geom = W.AttnGeometry(8, 2, 64)
    rng = np.random.default_rng(11)
    for n_new, split_q in [(1, 4), (4, 4), (40, 0)]:
        n = 300
        k = _rand(rng, n + n_new, 2, 64)
        v = _rand(rng, n + n_new, 2, 64) * 2.0 ** rng.integers(-60, 61, size=(n + n_new, 2, 1))
        v[::7] = 0
        q = _rand(rng, n + n_new, 8, 64)
        pool = _pool(geom, 32, 1, 32, split_q=split_q)
        a = [_bf16(t[:n]) for t in (q, k, v)]
        assert pool.replay(0, [0], [n], *a, torch.empty_like(a[0]), 0.125) == 0
        b = [_bf16(t[n:]) for t in (q, k, v)]
        o = torch.empty_like(b[0])
        assert pool.replay(0, [0], [n_new], *b, o, 0.125) == 0
        kk, vv = oracle.int8_read(k), oracle.int8_read(v)
        want = oracle.attention(q[n:], kk, vv, n, 0.125)
        mag = oracle.attention(q[n:], kk, np.abs(vv), n, 0.125)
        # prefill rounds q * scale as well: each score is off by at most 2^-8 sum |q k| scale
        smax = 0.125 * np.einsum("thd,nhd->thn", np.abs(q[n:]), np.abs(kk).repeat(4, 1)).max(-1)[..., None]
        rough = 2.0 ** -8 * (2.02 if n_new <= 8 else 2.02 + 2 * smax)
        assert (np.abs(_f64(o) - want) <= (rough + 2e-5) * (mag + np.abs(want))).all()


def test_fork_and_copy_on_write():
    """Branches of one base diverge from a shared partial block: codes and
    exponents are copied for every layer, the base keeps its own."""
    geom = W.AttnGeometry(8, 2, 64)
    rng = np.random.default_rng(21)
    pool, lone = _pool(geom, 40, 4, 8, n_layers=2), _pool(geom, 40, 1, 8, n_layers=2)
    base = [[_bf16(_rand(rng, 53, h, 64)) for h in (8, 2, 2)] for _ in range(2)]
    tails = [[[_bf16(_rand(rng, 21, h, 64)) for h in (8, 2, 2)] for _ in range(2)] for _ in range(2)]
    for p in (pool, lone):
        for layer in (0, 1):
            assert p.replay(layer, [0], [53], *base[layer], torch.empty_like(base[layer][0]), 0.1, commit=layer == 1) == 0
    before = [_stored(pool, layer, 0, 53) for layer in (0, 1)]
    assert pool.fork([0, 0], [1, 2]) == 0
    outs = []
    for layer in (0, 1):
        x = [torch.cat([tails[b][layer][i] for b in (0, 1)]) for i in range(3)]
        o = torch.empty_like(x[0])
        assert pool.replay(layer, [1, 2], [21, 21], *x, o, 0.1, commit=layer == 1) == 0
        outs.append(o)
    for layer in (0, 1):
        for a, b in zip(before[layer], _stored(pool, layer, 0, 53)):
            assert np.array_equal(a, b)
    for branch in (0, 1):
        assert lone.crop([0], [53]) == 0
        for layer in (0, 1):
            x = tails[branch][layer]
            o = torch.empty_like(x[0])
            assert lone.replay(layer, [0], [21], *x, o, 0.1, commit=layer == 1) == 0
            assert torch.equal(o, outs[layer][21 * branch:21 * branch + 21])
            for a, b in zip(_stored(lone, layer, 0, 74), _stored(pool, layer, 1 + branch, 74)):
                assert np.array_equal(a, b)


def test_single_tokens_of_forked_sequences():
    """Branches that share a partial block with their base and each other, re-decoded
    with a workspace (the first step copies the block, the next append in the decode
    kernel): as sequences that share nothing."""
    geom = W.AttnGeometry(8, 2, 128)
    rng = np.random.default_rng(41)
    base = [_bf16(_rand(rng, 53, h, 128)) for h in (8, 2, 2)]
    steps = [[_bf16(_rand(rng, 3, h, 128)) for h in (8, 2, 2)] for _ in range(14)]
    shared, own = (_pool(geom, 40, 3, 8, split_q=3, max_splits=4) for _ in range(2))
    assert shared.replay(0, [0], [53], *base, torch.empty_like(base[0]), 0.09) == 0
    assert shared.fork([0, 0], [1, 2]) == 0
    for i in range(3):
        assert own.replay(0, [i], [53], *base, torch.empty_like(base[0]), 0.09) == 0
    for n, x in enumerate(steps):
        o = [torch.empty_like(x[0]) for _ in range(2)]
        for pool, out in zip((shared, own), o):
            assert pool.replay(0, [0, 1, 2], [1, 1, 1], *x, out, 0.09) == 0
        assert torch.equal(o[0], o[1]), n
        for s in range(3):
            for a, b in zip(_stored(shared, 0, s, 54 + n), _stored(own, 0, s, 54 + n)):
                assert np.array_equal(a, b), (n, s)


def test_other_stream_and_captured_decode():
    """A decode step of two layers on a stream of its own, then recorded as a graph
    and replayed with other inputs and eager work between the replays."""
    geom = W.AttnGeometry(8, 2, 128)
    rng = np.random.default_rng(31)
    ctx = (400, 37, 1200)
    pool = _pool(geom, 140, 4, 90, n_layers=2, split_q=3, max_splits=32)
    tokens = [[_bf16(_rand(rng, sum(ctx), h, 128)) for h in (8, 2, 2)] for _ in range(2)]
    for layer in (0, 1):
        assert pool.replay(layer, [0, 1, 2], ctx, *tokens[layer], torch.empty_like(tokens[layer][0]), 0.09,
                           commit=layer == 1) == 0
    steps = [[_bf16(_rand(rng, 3, h, 128)) for h in (8, 2, 2)] for _ in range(4)]
    want = []
    for x in steps:
        o = [torch.empty_like(x[0]) for _ in range(2)]
        for layer in (0, 1):
            assert pool.replay(layer, [0, 1, 2], [1, 1, 1], *x, o[layer], 0.09, commit=False) == 0
        want.append(o)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o = torch.empty_like(steps[0][0])
    assert pool.replay(0, [0, 1, 2], [1, 1, 1], *steps[0], o, 0.09, commit=False, stream=side) == 0
    side.synchronize()
    assert torch.equal(o, want[0][0])
    x = [t.clone() for t in steps[0]]
    outs = [torch.empty_like(x[0]) for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for layer in (0, 1):
            assert pool.replay(layer, [0, 1, 2], [1, 1, 1], *x, outs[layer], 0.09, commit=False) == 0
    for i in (0, 2, 1, 3, 0):
        for a, b in zip(x, steps[i]):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[i][0]) and torch.equal(outs[1], want[i][1])
        eager = torch.empty_like(x[0])
        assert pool.replay(1, [2], [1], *(t[2:] for t in steps[3 - i % 2]), eager[:1], 0.09, commit=False) == 0
        torch.cuda.synchronize()


def test_static_scratch_equals_the_workspace():
    geom = W.AttnGeometry(32, 8, 128)
    from paper_2609_04875_amd import workspace_bytes
    rng = np.random.default_rng(41)
    ws = workspace_bytes(32, 128, 40, 16)
    a, b = _pool(geom, 80, 1, 80, split_q=40), _pool(geom, 80, 1, 80)
    x = [_bf16(_rand(rng, 1000, h, 128)) for h in (32, 8, 8)]
    for p in (a, b):
        assert p.replay(0, [0], [1000], *x, torch.empty_like(x[0]), 0.09) == 0
    for n in (40, 1):
        y = [_bf16(_rand(rng, n, h, 128)) for h in (32, 8, 8)]
        oa, ob = torch.empty_like(y[0]), torch.empty_like(y[0])
        assert a.replay(0, [0], [n], *y, oa, 0.09, commit=False) == 0
        assert b.replay_static(0, [0], [n], *y, ob, 0.09, ws, commit=False) == 0
        assert torch.equal(oa, ob)


def test_caches_past_32_bits():
    """Blocks at the end of a cache of more than 2^32 codes: prefill (four-wave,
    pipelined, through the copy) and decode as in a small pool."""
    from paper_2609_04875_amd import INT8, KVPool
    geom, n_blocks = W.AttnGeometry(32, 8, 128), 270000
    log(f"int8 cache of {n_blocks * 16384:.2e} codes")
    rng = np.random.default_rng(61)
    order = list(range(n_blocks))                                # pops yield the last ids first
    far = KVPool(1, 32, 8, 128, n_blocks, 1, 256, INT8, 16, order, workspace_bytes=64 << 20)
    near = KVPool(1, 32, 8, 128, 256, 1, 256, INT8, 16, workspace_bytes=64 << 20)
    a = [_bf16(_rand(rng, 45, h, 128)) for h in (32, 8, 8)]
    b = [_bf16(_rand(rng, 2070, h, 128)) for h in (32, 8, 8)]
    c = [_bf16(_rand(rng, 1, h, 128)) for h in (32, 8, 8)]
    outs = []
    for pool in (far, near):
        for kernel in ("four_wave", "pipelined", "auto"):
            pool.set_prefill_kernel(kernel)
            if pool.seq_len(0):
                assert pool.crop([0], [0]) == 0
            for x in (a, b, c):
                outs.append(torch.empty_like(x[0]))
                assert pool.replay(0, [0], [len(x[0])], *x, outs[-1], 0.09) == 0
    assert int(far.block_tables[0, :120].min()) > 262144          # past 2^32 bytes of codes
    assert all(torch.equal(x, y) for x, y in zip(outs[:9], outs[9:]))


@pytest.mark.parametrize("hq,hkv,B,P,S", [(32, 8, 16, 3000, 700), (32, 8, 32, 1990, 1024), (32, 4, 64, 2500, 250),
                                          (16, 16, 16, 4001, 1500), (8, 2, 16, 900, 701)])
def test_split_prefill_through_the_copy(hq, hkv, B, P, S):
    """Calls with split keys on the bf16 copy behind the partials: the bits of the
    pipelined kernel on the codes, of a pool whose workspace has no room for the copy,
    and the oracle's values."""
    from paper_2609_04875_amd import INT8, KVPool, workspace_bytes
    log(f"int8 split prefill {hq}/{hkv} B={B} {S} on {P}")
    geom, rng = W.AttnGeometry(hq, hkv, 128), np.random.default_rng(S)
    z = [_bf16(_rand(rng, P, h, 128)) for h in (hq, hkv, hkv)]
    x = [_bf16(_rand(rng, S, h, 128)) for h in (hq, hkv, hkv)]
    copy = 512 * hkv * (P + S + 16) + 4 * (P + S)
    outs = []
    for splits, room, kind in ((8, 0, "pipelined"), (8, copy, "auto"), (8, copy, "pipelined")):
        pool = KVPool(1, hq, hkv, 128, _blocks(P + S, B), 1, _blocks(P + S, B), INT8, B,
                      workspace_bytes=workspace_bytes(hq, 128, S, splits) + room)
        pool.set_prefill_kernel(kind)
        assert pool.replay(0, [0], [P], *z, torch.empty_like(z[0]), 0.09) == 0
        outs.append(torch.full_like(x[0], float("nan")))
        assert pool.replay(0, [0], [S], *x, outs[-1], 0.09) == 0
        torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    k, v = _read(pool, 0, 0, P + S)
    rows = np.unique(np.r_[0, 1, S - 1, rng.integers(0, S, 12)])
    for i in rows:
        q = _f64(x[0][i:i + 1])
        want = oracle.attention(q, k[:P + i + 1], v[:P + i + 1], P + int(i), 0.09)
        assert (np.abs(_f64(outs[1][i:i + 1]) - want) <= _decode_bound(q, k[:P + i + 1], v[:P + i + 1], P + int(i), 0.09, want)
                + _query_rounding(q[0], k[:P + i + 1], v[:P + i + 1], 0.09, want[0])).all()


@pytest.mark.parametrize("hq,hkv,d,B,P,S", [
    (8, 8, 64, 32, (2100, 700, 1500), (40, 120, 65)), (8, 2, 64, 16, (1000, 0, 3000), (300, 64, 170)),
    (16, 4, 64, 64, (2600,), (37,)), (28, 4, 128, 16, (2100, 900), (12, 40)), (32, 8, 128, 64, (3001,), (9,)),
    (8, 8, 64, 16, (700, 650), (300, 280))])
def test_split_prefill_matches_the_oracle(hq, hkv, d, B, P, S):
    """Prefill calls with split keys, few rows (joined by a wave each at head_dim 64) and
    more, over a workspace of NaN: every partial that is read was written by the call."""
    log(f"int8 split prefill {hq}/{hkv}/{d} B={B} {S} on {P}")
    geom, rng, n = W.AttnGeometry(hq, hkv, d), np.random.default_rng(P[0] + S[0]), len(P)
    pool = _pool(geom, sum(_blocks(p + s, B) for p, s in zip(P, S)), n, max(_blocks(p + s, B) for p, s in zip(P, S)), B,
                 split_q=sum(S), max_splits=16)
    for i, p in enumerate(P):
        z = [_bf16(_rand(rng, p, h, d)) for h in (hq, hkv, hkv)]
        assert pool.replay(0, [i], [p], *z, torch.empty_like(z[0]), 0.1) == 0
    x = [_bf16(_rand(rng, sum(S), h, d)) for h in (hq, hkv, hkv)]
    o = [torch.full_like(x[0], float("nan")) for _ in range(2)]
    for out in o:
        pool.workspace.fill_(0xFF)
        assert pool.replay(0, list(range(n)), S, *x, out, 0.1, commit=out is o[1]) == 0
        torch.cuda.synchronize()
    assert torch.equal(o[0], o[1]) and (pool.workspace[:1024] != 0xFF).any()        # there were splits
    off = 0
    for i, (p, s) in enumerate(zip(P, S)):
        k, v = _read(pool, 0, i, p + s)
        for t in np.unique(np.r_[0, s - 1, rng.integers(0, s, 6)]):
            q = _f64(x[0][off + t:off + t + 1])
            kk, vv = k[:p + t + 1], v[:p + t + 1]
            want = oracle.attention(q, kk, vv, p + int(t), 0.1)
            bound = _decode_bound(q, kk, vv, p + int(t), 0.1, want) + _query_rounding(q[0], kk, vv, 0.1, want[0])
            assert (np.abs(_f64(o[0][off + t:off + t + 1]) - want) <= bound).all(), (i, t)
        off += s


def test_captured_prefill_through_the_copy():
    """A long suffix recorded with its copy in the workspace, replayed with other
    inputs and eager calls that use the same workspace in between."""
    geom = W.AttnGeometry(8, 2, 128)
    rng = np.random.default_rng(71)
    pool = _pool(geom, 300, 1, 300, split_q=200, max_splits=16)
    z = [_bf16(_rand(rng, 700, h, 128)) for h in (8, 2, 2)]
    assert pool.replay(0, [0], [700], *z, torch.empty_like(z[0]), 0.09) == 0
    n = 64 * 140
    pool2 = _pool(geom, 700, 1, 700, split_q=n, max_splits=2)
    assert pool2.replay(0, [0], [700], *z, torch.empty_like(z[0]), 0.09) == 0
    xs = [[torch.randn(n, h, 128, device="cuda").to(torch.bfloat16) for h in (8, 2, 2)] for _ in range(3)]
    want = []
    for x in xs:
        want.append(torch.empty_like(x[0]))
        pool2.workspace.fill_(0xA5)
        assert pool2.replay(0, [0], [n], *x, want[-1], 0.09, commit=False) == 0
        torch.cuda.synchronize()
        assert (pool2.workspace[:4096] != 0xA5).any()                # the copy was made
    held, out = [t.clone() for t in xs[0]], torch.empty_like(want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert pool2.replay(0, [0], [n], *held, out, 0.09, commit=False) == 0
    for i in (0, 2, 1, 0):
        for p, q in zip(held, xs[i]):
            p.copy_(q)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i])
        one = [t[:1].clone() for t in xs[1]]
        assert pool2.replay(0, [0], [1], *one, torch.empty_like(one[0]), 0.09, commit=False) == 0
        torch.cuda.synchronize()


def test_refusals_change_nothing():
    import ctypes
    from paper_2609_04875_amd import BF16, EINVAL, INT8, KVPool
    from paper_2609_04875_amd import _native as N
    geom = W.AttnGeometry(4, 2, 64)
    pool, plain = _pool(geom, 8, 1, 8), KVPool(1, 4, 2, 64, 8, 1, 8, BF16)
    assert N.lib.pgsr_pool_set_kv_exponents(plain._h, pool.kv_exponents.data_ptr()) == EINVAL
    assert N.lib.pgsr_pool_set_kv_exponents(pool._h, None) == EINVAL
    assert N.lib.pgsr_pool_set_kv_exponents(pool._h, pool.kv_exponents.data_ptr() + 8) == EINVAL
    with pytest.raises(N.PgsrError):
        pool.set_kv_scales([1.0], [1.0])                           # per-layer scales are the FP8 pool's
    x = [torch.ones(5, h, 64, dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2)]
    # a pool made through the C ABI, whose exponents were never given
    h = ctypes.c_void_p()
    t = pool
    N.check(N.lib.pgsr_pool_create(1, 4, 2, 64, 16, INT8, 8, 1, 8, t.k_cache.data_ptr(), t.v_cache.data_ptr(),
                                   t.block_tables.data_ptr(), t.seq_lens.data_ptr(), t.free_list.data_ptr(),
                                   t.free_top.data_ptr(), t.ref_counts.data_ptr(), None, 0, None, None, ctypes.byref(h)))
    o = torch.full_like(x[0], 7.0)
    one = N.int32_array([0])
    assert N.lib.pgsr_replay_prefill(h, 0, 1, one, N.int32_array([5]), x[0].data_ptr(), x[1].data_ptr(), x[2].data_ptr(),
                                     o.data_ptr(), 0.1, 1, None, None) == EINVAL
    torch.cuda.synchronize()
    assert (o == 7).all() and int(t.free_top.item()) == 8 and not t.k_cache.any()
    N.lib.pgsr_pool_destroy(h)
    with pytest.raises(ValueError):
        pool.replay(0, [0], [5], *(y.to(torch.int8) for y in x), o, 0.1)


# calls that fill the chip without splits and read each key in five tiles or more:
# geometry, block size, prefixes, suffixes
EXPAND = [
    (W.AttnGeometry(32, 8, 128), 16, (1001,), (2100,)),
    (W.AttnGeometry(32, 8, 128), 64, (277, 100, 640, 315), (1900, 1700, 513, 300)),
    (W.AttnGeometry(28, 4, 128), 32, (250, 31, 16), (1400, 900, 1500)),
    (W.AttnGeometry(8, 1, 128), 16, tuple(range(503, 635, 2)), (416,) * 66),
]


@pytest.mark.parametrize("case", range(len(EXPAND)))
def test_prefill_through_a_bf16_copy_has_the_same_bits(case):
    """A workspace with the room for the copy, one a byte short of it and none: the
    copy is made exactly where it fits, and the bits never differ."""
    geom, B, P, S = EXPAND[case]
    log(f"int8 prefill through a copy, case {case}")
    C, d = [p + 40 for p in P], geom.head_dim
    nb = sum(_blocks(max(c, p + s), B) + 1 for p, s, c in zip(P, S, C))
    bps = max(_blocks(max(c, p + s), B) for p, s, c in zip(P, S, C)) + 1
    data, _ = _episodes(np.random.default_rng(70 + case), geom, P, S, C, False)
    # what the last launch's entries need (64 at most): two caches of 16-token blocks and a table
    last = [(p + s) for p, s in zip(P, S)][len(P) - (len(P) - 1) % 64 - 1:]
    need = lambda kv: (2 * 2 * 16 * d * geom.n_kv_heads * sum(_blocks(x) for x in kv)  # noqa: E731
                       + 4 * len(kv) * max(_blocks(x) for x in kv))
    first = [(p + s) for p, s in zip(P, S)][:64]
    from paper_2609_04875_amd import INT8, KVPool
    outs, used = [], []
    for ws in (0, need(first) - 1, need(first)):
        pool = KVPool(1, geom.n_q_heads, geom.n_kv_heads, d, nb, len(P), bps, INT8, B, workspace_bytes=ws)
        q, k, v, cq, ck, cv = data
        seqs = list(range(len(P)))
        assert pool.replay(0, seqs, C, cq, ck, cv, torch.empty_like(cq), 0.09) == 0
        assert pool.crop(seqs, P, poison=True) == 0
        if ws:
            pool.workspace.fill_(0xA5)
        o = torch.full_like(q, float("nan"))
        assert pool.replay(0, seqs, S, q, k, v, o, 0.09) == 0
        torch.cuda.synchronize()
        outs.append(o)
        used.append(bool(ws) and bool((pool.workspace[:4096] != 0xA5).any()))
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    assert torch.isfinite(outs[0]).all()
    assert used[2] and (len(P) > 64 or not used[1])
