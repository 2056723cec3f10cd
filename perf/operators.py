"""The 8-bit integer operators as cases that can be timed: the KV cache of int8
codes with an exponent for each token and head, and the int8 product with a
scale for each token and channel.

A case is a dict of plain values.  ``prepare`` makes what a program has in hand
before the call (inputs on the GPU, the cached sequences, quantised weights),
``run`` is one pass, ``exact`` the same result in 64 bits from the definitions.
The kinds:

* ``cache``: one attention layer that is not the last, over a paged cache held
  in int8: the new tokens of each sequence are quantised and appended, then
  attend (``KVPool(dtype=INT8).replay`` without commit).  One new token for each
  is a re-decode step, more are a replayed suffix.  The result is what the new
  tokens' queries see; a program reads the appended keys and values in no other
  way, and a new token weighs enough in its own query's result to show there.
* ``linear``: an int8 product whose left operand is quantised a token at a time
  within the call: from bf16 states (``quantize_rows``), through RMSNorm
  (``rmsnorm_int8``) or through the SwiGLU product (``silu_mul_int8``), then
  ``gemm_int8``, or ``gemm_int8_multi`` for a layer's Q, K and V projections.

``own`` chooses between the plain form (elementary torch operations in 32 bits)
and the framework's calls.
"""
from __future__ import annotations

import math

import torch

own = False

GEOMETRY = {            # query heads, KV heads, head size, d_model, d_ff
    "8b": (32, 8, 128, 4096, 14336),
    "70b": (64, 8, 128, 8192, 28672),
    "7b_g7": (28, 4, 128, 3584, 18944),
    "mha8_d64": (8, 8, 64, 512, 1408),
}
EPS = 1e-5
E_LO, E_HI = -100, 100      # exponents of a cached row


def listed():
    return [
        # one re-decoded token of a session of the paper's length: latency decides
        {"name": "cache_decode_1", "kind": "cache", "geometry": "8b", "seqs": 1, "ctx_lo": 1330, "ctx_hi": 1330,
         "new_lo": 1, "new_hi": 1, "block": 16, "len_seed": 0},
        # re-decode of 32 sessions in step, 8192 tokens cached for each
        {"name": "cache_decode_b32_8k", "kind": "cache", "geometry": "8b", "seqs": 32, "ctx_lo": 8192, "ctx_hi": 8192,
         "new_lo": 1, "new_hi": 1, "block": 16, "len_seed": 0},
        # sessions of very different lengths, seven query heads to a KV head
        {"name": "cache_decode_b40_ragged_g7", "kind": "cache", "geometry": "7b_g7", "seqs": 40, "ctx_lo": 500,
         "ctx_hi": 16000, "new_lo": 1, "new_hi": 1, "block": 16, "len_seed": 4},
        # the benchmark's episode: 8189 tokens kept (inside a block), 2048 replayed
        {"name": "cache_replay_8b", "kind": "cache", "geometry": "8b", "seqs": 1, "ctx_lo": 8189, "ctx_hi": 8189,
         "new_lo": 2048, "new_hi": 2048, "block": 16, "len_seed": 0},
        # a batch of short suffixes on the small heads of 64, blocks of 32 tokens
        {"name": "cache_replay_b7_ragged_d64", "kind": "cache", "geometry": "mha8_d64", "seqs": 7, "ctx_lo": 100,
         "ctx_hi": 3000, "new_lo": 40, "new_hi": 500, "block": 32, "len_seed": 5},
        # one token through a layer's Q, K and V projections behind the norm: weights are read once
        {"name": "linear_qkv_1", "kind": "linear", "front": "norm", "m": 1, "k": 4096, "n": 4096, "n2": 1024,
         "residual": False},
        # 32 sessions in step through the gate|up projection
        {"name": "linear_gate_up_32", "kind": "linear", "front": "norm", "m": 32, "k": 4096, "n": 28672, "n2": 0,
         "residual": False},
        # the paper's short suffix through the down projection of the group-of-seven model
        {"name": "linear_down_102_g7", "kind": "linear", "front": "gate", "m": 102, "k": 18944, "n": 3584, "n2": 0,
         "residual": True},
        # sizes that fill no tile and no K step
        {"name": "linear_odd", "kind": "linear", "front": "rows", "m": 333, "k": 1232, "n": 1000, "n2": 0,
         "residual": True},
        # the benchmark's suffix through the gate|up projection
        {"name": "linear_gate_up_2048", "kind": "linear", "front": "norm", "m": 2048, "k": 4096, "n": 28672, "n2": 0,
         "residual": False},
        # the same suffix through the down projection
        {"name": "linear_down_2048", "kind": "linear", "front": "gate", "m": 2048, "k": 14336, "n": 4096, "n2": 0,
         "residual": True},
        # a long suffix through the output projection of the 70B-like layers
        {"name": "linear_out_8192_70b", "kind": "linear", "front": "rows", "m": 8192, "k": 8192, "n": 8192, "n2": 0,
         "residual": True},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "replay", "replay", "linear", "linear", "linear"])
    if kind == "decode":
        seqs = _log_int(rng, 1, 60)
        ctx = _log_int(rng, 1, min(30000, 250000 // seqs))
        return {"kind": "cache", "geometry": rng.choice(["8b", "8b", "70b", "7b_g7", "mha8_d64"]), "seqs": seqs,
                "ctx_lo": max(0, int(ctx * rng.uniform(0.1, 1.0))), "ctx_hi": ctx, "new_lo": 1,
                "new_hi": rng.choice([1, 1, 1, 3]), "block": rng.choice([16, 16, 32, 64]),
                "len_seed": rng.randrange(1000)}
    if kind == "replay":
        geometry = rng.choice(["8b", "8b", "70b", "7b_g7", "mha8_d64"])
        seqs = rng.choice([1, 1, _log_int(rng, 2, 8)])
        new = _log_int(rng, 2, 2000 // seqs)
        ctx = _log_int(rng, 1, (9000 if geometry != "70b" else 5000) // (1 if seqs == 1 else 3))
        return {"kind": "cache", "geometry": geometry, "seqs": seqs, "ctx_lo": rng.choice([0, ctx // 3, ctx]),
                "ctx_hi": ctx, "new_lo": max(1, int(new * rng.uniform(0.2, 1.0))), "new_hi": new,
                "block": rng.choice([16, 16, 32, 64]), "len_seed": rng.randrange(1000)}
    front = rng.choice(["rows", "norm", "gate"])
    m = _log_int(rng, 1, 6000)
    if rng.random() < 0.5:
        _, _, _, dm, dff = GEOMETRY[rng.choice(sorted(GEOMETRY))]
        k, n = {"rows": (dm, dm), "norm": (dm, 2 * dff), "gate": (dff, dm)}[front]
    else:
        k, n = 16 * _log_int(rng, 1, 1000), 8 * _log_int(rng, 1, 2000)
    m = max(1, min(m, int(4e11 / (n * k))))
    n2 = 8 * _log_int(rng, 1, 200) if front == "norm" and rng.random() < 0.3 else 0
    return {"kind": "linear", "front": front, "m": m, "k": k, "n": n, "n2": n2,
            "residual": n2 == 0 and rng.random() < 0.5}


def _lengths(case):
    """Cached and new tokens of each sequence."""
    g = torch.Generator().manual_seed(case["len_seed"])
    pick = lambda lo, hi: torch.randint(lo, hi + 1, (case["seqs"],), generator=g).tolist()  # noqa: E731
    return pick(case["ctx_lo"], case["ctx_hi"]), pick(case["new_lo"], case["new_hi"])


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _power(e):
    """2^e in fp32, exactly (a library power may be off by a rounding, and ties are common here)."""
    return ((e + 127) << 23).view(torch.float32)


def _quantize_cache_rows(x):
    """Codes (int8) and exponents (int32) of rows of the last axis, from the definition."""
    x = x.float()
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.frexp(amax).exponent - 7          # floor(log2) - 6
    e = torch.where(amax > 0, e, torch.full_like(e, E_LO)).clamp(E_LO, E_HI)
    codes = torch.round(x * _power(-e)).clamp(-127, 127).to(torch.int8)
    return codes, e.squeeze(-1)


def _quantize_rows(x):
    """Codes (held in fp32) and scales of the rows of x (fp32): a scale for each."""
    s = x.abs().amax(-1, keepdim=True) / 127.0
    codes = torch.where(s > 0, torch.round(x / torch.where(s > 0, s, torch.ones_like(s))), torch.zeros_like(x))
    return codes, s.squeeze(-1)


def _draw_kv(case, seed):
    """Packed bf16 K, V of every token (cached, then new, a sequence after the other) and the q of the new ones."""
    hq, hkv, d, _, _ = GEOMETRY[case["geometry"]]
    ctx, new = _lengths(case)
    g = _gen(seed)
    n = sum(ctx) + sum(new)
    # keys with channels of different size, tokens of different size; a new token looks at itself more than at others
    channel = torch.exp(0.4 * torch.randn(hkv, d, device="cuda", generator=g))
    channel = channel / channel.square().mean().sqrt()
    size = torch.exp(0.25 * torch.randn(n, 1, 1, device="cuda", generator=g))
    k = (torch.randn(n, hkv, d, device="cuda", generator=g) * channel * size).to(torch.bfloat16)
    v = (torch.randn(n, hkv, d, device="cuda", generator=g) * size).to(torch.bfloat16)
    starts, is_new = 0, []
    for c, s in zip(ctx, new):
        is_new += range(starts + c, starts + c + s)
        starts += c + s
    is_new = torch.tensor(is_new, device="cuda")
    q = torch.randn(len(is_new), hq, d, device="cuda", generator=g)
    q = (q + 0.6 * k[is_new].float().repeat_interleave(hq // hkv, 1)).to(torch.bfloat16)
    return k, v, q, is_new


def prepare(case, seed):
    if case["kind"] == "linear":
        m, n, n2, k = (case[x] for x in ("m", "n", "n2", "k"))
        g = _gen(seed)
        width = 2 * k if case["front"] == "gate" else k
        channel = torch.exp(0.5 * torch.randn(width, device="cuda", generator=g))   # a few large channels
        st = {"case": case, "x": (torch.randn(m, width, device="cuda", generator=g) * channel).to(torch.bfloat16),
              "w": [], "r": None, "gain": None}
        for rows in (n, n2, n2) if n2 else (n,):
            w = torch.randn(rows, k, device="cuda", generator=g) * k ** -0.5
            codes, scales = _quantize_rows(w)
            st["w"].append((codes.to(torch.int8), scales))
        if case["front"] == "norm":
            st["gain"] = (1 + 0.1 * torch.randn(k, device="cuda", generator=g)).to(torch.bfloat16)
        if case["residual"]:
            st["r"] = torch.randn(m, n, device="cuda", generator=g).to(torch.bfloat16)
        st["out"] = [torch.empty(m, w.shape[0], dtype=torch.bfloat16, device="cuda") for w, _ in st["w"]]
        return st
    hq, hkv, d, _, _ = GEOMETRY[case["geometry"]]
    ctx, new = _lengths(case)
    k, v, q, is_new = _draw_kv(case, seed)
    old = torch.ones(k.shape[0], dtype=torch.bool, device="cuda")
    old[is_new] = False
    ck, cv = k[old], v[old]
    st = {"case": case, "q": q, "k": k[is_new].contiguous(), "v": v[is_new].contiguous(), "new": new, "ctx": ctx,
          "seqs": list(range(len(ctx)))}
    if own:
        from paper_2609_04875_amd import INT8, KVPool, workspace_bytes
        block = case["block"]
        row = max(-(-(c + s) // block) for c, s in zip(ctx, new))
        pool = KVPool(1, hq, hkv, d, sum(-(-(c + s) // block) for c, s in zip(ctx, new)), len(ctx), row, INT8, block,
                      workspace_bytes=workspace_bytes(hq, d, sum(new), 64 if max(new) <= 4 else 16))
        at = 0
        for i, c in enumerate(ctx):          # the cached sessions, a chunk at a time
            for t in range(0, c, 4096):
                s = min(4096, c - t)
                z = torch.zeros(s, hq, d, dtype=torch.bfloat16, device="cuda")
                rc = pool.replay(0, [i], [s], z, ck[at:at + s], cv[at:at + s], torch.empty_like(z), 1.0)
                if rc:
                    raise RuntimeError(f"replay of the cached tokens: status {rc}")
                at += s
        st["pool"], st["out"] = pool, torch.empty_like(q)
        return st
    # the plain cache: codes and exponents of every sequence, padded to the longest
    n, longest = len(ctx), max(c + s for c, s in zip(ctx, new))
    seq_old = torch.repeat_interleave(torch.arange(n), torch.tensor(ctx)).cuda()
    pos_old = torch.cat([torch.arange(c) for c in ctx]).cuda()
    st["seq"] = torch.repeat_interleave(torch.arange(n), torch.tensor(new)).cuda()
    st["tok"] = torch.cat([torch.arange(s) for s in new]).cuda()
    st["pos"] = torch.cat([torch.arange(c, c + s) for c, s in zip(ctx, new)]).cuda()
    for name, x in (("k", ck), ("v", cv)):
        st["codes_" + name] = torch.zeros(n, longest, hkv, d, dtype=torch.int8, device="cuda")
        st["exps_" + name] = torch.zeros(n, longest, hkv, dtype=torch.int32, device="cuda")
        st["codes_" + name][seq_old, pos_old], st["exps_" + name][seq_old, pos_old] = _quantize_cache_rows(x)
    return st


def _cache_plain(st):
    hq, hkv, d, _, _ = GEOMETRY[st["case"]["geometry"]]
    n, most, G = len(st["ctx"]), max(st["new"]), hq // hkv
    seq, tok, pos = st["seq"], st["tok"], st["pos"]
    kv = []
    for name in ("k", "v"):
        st["codes_" + name][seq, pos], st["exps_" + name][seq, pos] = _quantize_cache_rows(st[name])
        x = st["codes_" + name].float() * _power(st["exps_" + name]).unsqueeze(-1)
        kv.append(x.transpose(1, 2).contiguous())                        # [n, hkv, keys, d]
    q = torch.zeros(n, most, hq, d, device="cuda")
    at = torch.full((n, most), -1, dtype=torch.int64, device="cuda")     # position of each query, -1: none
    q[seq, tok], at[seq, tok] = st["q"].float(), pos
    q = q.view(n, most, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, most * G, d)
    s = torch.matmul(q, kv[0].transpose(-1, -2).contiguous()) * d ** -0.5
    keys = torch.arange(s.shape[-1], device="cuda")
    seen = (keys <= at.repeat_interleave(G, 1).unsqueeze(-1)).unsqueeze(1)
    s = torch.where(seen, s, torch.full_like(s, -torch.inf))
    s = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-3e38))
    o = torch.matmul(s, kv[1]) / s.sum(-1, keepdim=True).clamp(min=1e-38)
    o = o.view(n, hkv, most, G, d).permute(0, 2, 1, 3, 4).reshape(n, most, hq, d)
    return o[seq, tok].to(torch.bfloat16)


def _linear_plain(st):
    x, front = st["x"].float(), st["case"]["front"]
    if front == "norm":
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * st["gain"].float()
    elif front == "gate":
        gate, up = x.chunk(2, -1)
        x = gate / (1 + torch.exp(-gate)) * up
    codes, scales = _quantize_rows(x)
    outs = [torch.matmul(codes, wq.float().t()) * (scales[:, None] * ws) for wq, ws in st["w"]]
    if st["r"] is not None:
        outs[0] = outs[0] + st["r"].float()
    return [y.to(torch.bfloat16) for y in outs]


def run(st):
    if st["case"]["kind"] == "cache":
        if not own:
            return _cache_plain(st)
        rc = st["pool"].replay(0, st["seqs"], st["new"], st["q"], st["k"], st["v"], st["out"],
                               st["q"].shape[-1] ** -0.5, commit=False)
        if rc:
            raise RuntimeError(f"replay: status {rc}")
        return st["out"]
    if not own:
        return _linear_plain(st)
    from paper_2609_04875_amd import gemm_int8, gemm_int8_multi, quantize_rows, rmsnorm_int8, silu_mul_int8
    front = st["case"]["front"]
    if front == "norm":
        xq, xs = rmsnorm_int8(st["x"], st["gain"], EPS)
    elif front == "gate":
        xq, xs = silu_mul_int8(st["x"])
    else:
        xq, xs = quantize_rows(st["x"])
    if len(st["w"]) > 1:
        return gemm_int8_multi(xq, xs, [w for w, _ in st["w"]], [s for _, s in st["w"]], st["out"])
    (wq, ws), = st["w"]
    return [gemm_int8(xq, xs, wq, ws, r=st["r"], out=st["out"][0])]


def work(case):
    if case["kind"] == "linear":
        m, k, n = case["m"], case["k"], case["n"] + 2 * case["n2"]
        b = 2 * m * k * (2 if case["front"] == "gate" else 1) + n * k + 4 * n + 2 * m * n
        b += 2 * k * (case["front"] == "norm") + 2 * m * n * case["residual"]
        return {"bytes": b, "flops": 2 * m * n * k}
    hq, hkv, d, _, _ = GEOMETRY[case["geometry"]]
    ctx, new = _lengths(case)
    pairs = sum(s * c + s * (s + 1) // 2 for c, s in zip(ctx, new))
    token = 2 * hkv * (d + 1)                          # codes and exponents of a token's K and V
    b = sum(ctx) * token + sum(new) * (2 * hq * d * 2 + 2 * hkv * d * 2 + token)
    return {"bytes": b, "flops": 4 * hq * d * pairs}


def exact(case, seed):
    if case["kind"] == "linear":
        return _linear_exact(case, seed)
    hq, hkv, d, _, _ = GEOMETRY[case["geometry"]]
    ctx, new = _lengths(case)
    k, v, q, _ = _draw_kv(case, seed)
    read = []
    for x in (k.double(), v.double()):                 # what the cache gives back: code * 2^e
        # exponents from and into the bits of fp64: many values are exact ties, which a power off by a rounding moves
        e = ((x.abs().amax(-1, keepdim=True).view(torch.int64) >> 52) - 1023 - 6).clamp(-100, 100)
        step = ((e + 1023) << 52).view(torch.float64)
        read.append((x / step).round().clamp(-127, 127) * step)
    out, at, row = [], 0, 0
    for c, s in zip(ctx, new):                         # a sequence and a KV head at a time
        heads = []
        for h in range(hkv):
            kk, vv = (x[at:at + c + s, h] for x in read)
            qq = q[row:row + s, h * (hq // hkv):(h + 1) * (hq // hkv)].double()
            w = torch.einsum("sgd,ld->sgl", qq, kk) / math.sqrt(d)
            late = torch.arange(c + s, device="cuda")[None] > torch.arange(c, c + s, device="cuda")[:, None]
            w.masked_fill_(late[:, None, :], -math.inf)
            heads.append(torch.einsum("sgl,ld->sgd", torch.softmax(w, -1), vv))
        out.append(torch.cat(heads, 1))
        at, row = at + c + s, row + s
    return torch.cat(out)


def _linear_exact(case, seed):
    st = prepare(case, seed)
    x = st["x"].double()
    if case["front"] == "norm":
        x = x / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * st["gain"].double()
    elif case["front"] == "gate":
        half = x.shape[1] // 2
        x = torch.sigmoid(x[:, :half]) * x[:, :half] * x[:, half:]
    step = x.abs().max(-1, keepdim=True).values / 127
    codes = torch.nan_to_num((x / step).round())
    outs = [(codes @ wq.double().T) * step * ws.double() for wq, ws in st["w"]]
    if st["r"] is not None:
        outs[0] += st["r"].double()
    return outs
