"""Full decoder-layer replay: F of Eq. (1) at the real geometries.

Per layer (pre-norm, as in the public architecture of the model families the
paper runs): h = RMSNorm(x) g_attn; Q, K, V = h Wq, h Wk, h Wv; rotary
embedding of Q and K at the tokens' absolute positions (a replay from P
rotates exactly as the full run); attention through the paged pool (one pool
layer per model layer); x <- x + O Wo; h2 = RMSNorm(x) g_mlp;
x <- x + (SiLU(h2 Wg) * (h2 Wu)) Wd.  Every step is a library call; this
module only sequences them and owns scratch tensors.

Weights may be int8 codes with a scale for each output channel
(``quantize_weights``): the projections then run on 8-bit integers, their left
operands quantised a token at a time behind the norms, the attention and the
gate.  The cache may be int8 or FP8 whatever the weights are.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Sequence, Tuple, Union

import torch

from . import _native as N
from .int8 import gemm_int8, gemm_int8_multi, quantize_rows, rmsnorm_int8, silu_mul_int8
from .pool import KVPool, _dev_ptr, gemm_bf16, gemm_bf16_multi, gemm_silu_bf16

PROJECTIONS = ("wq", "wk", "wv", "wo", "w_gate_up", "w_down")
Weight = Union[torch.Tensor, Tuple[torch.Tensor, torch.Tensor]]


def quantize_weights(weights: Sequence[Dict[str, torch.Tensor]]) -> List[Dict[str, Weight]]:
    """The weights of ``DecoderReplay`` with every projection as int8 codes and a
    fp32 scale for each output channel; the gains stay bf16."""
    return [{name: quantize_rows(w) if name in PROJECTIONS else w for name, w in layer.items()} for layer in weights]


def _stream(stream):
    return (stream or torch.cuda.current_stream()).cuda_stream


def rmsnorm(x: torch.Tensor, gain: torch.Tensor, eps: float, out: Optional[torch.Tensor] = None, stream=None):
    out = torch.empty_like(x) if out is None else out
    N.check(N.lib.pgsr_rmsnorm_bf16(x.shape[0], x.shape[1], x.data_ptr(), gain.data_ptr(), float(eps),
                                    out.data_ptr(), _stream(stream)))
    return out


def rope_(x: torch.Tensor, positions: torch.Tensor, theta: float, stream=None) -> torch.Tensor:
    """In place on x [n, heads, d]; positions: int32 [n] on the GPU."""
    assert positions.dtype == torch.int32 and positions.is_cuda
    N.check(N.lib.pgsr_rope_bf16(x.shape[0], x.shape[1], x.shape[2], x.data_ptr(), positions.data_ptr(),
                                 float(theta), _stream(stream)))
    return x


def rope_qk_(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, theta: float, stream=None) -> None:
    """``rope_`` of q [n, n_q_heads, d] and k [n, n_kv_heads, d] in one launch."""
    n, hq, d = q.shape
    if tuple(k.shape[::2]) != (n, d) or positions.numel() < n:
        raise ValueError(f"q is {tuple(q.shape)}, k {tuple(k.shape)}, positions {tuple(positions.shape)}")
    dv = q.device.index
    qp, kp = (_dev_ptr(t, torch.bfloat16, name, dv, n * t.shape[1] * d) for t, name in ((q, "q"), (k, "k")))
    N.check(N.lib.pgsr_rope_qk_bf16(n, hq, k.shape[1], d, qp, kp, _dev_ptr(positions, torch.int32, "positions", dv),
                                    float(theta), _stream(stream)))


def silu_mul(gate_up: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    n, two_ff = gate_up.shape
    out = torch.empty((n, two_ff // 2), dtype=gate_up.dtype, device=gate_up.device) if out is None else out
    N.check(N.lib.pgsr_silu_mul_bf16(n, two_ff // 2, gate_up.data_ptr(), out.data_ptr(), _stream(stream)))
    return out


class DecoderReplay:
    def __init__(self, weights: Sequence[Dict[str, Weight]], n_q_heads: int, n_kv_heads: int,
                 head_dim: int, eps: float, theta: float, n_blocks: int, max_seqs: int,
                 max_blocks_per_seq: int, block_size: int = 16, workspace_bytes: int = 0,
                 kv_dtype: int = N.BF16):
        """``weights``: per layer a dict of bf16 CUDA tensors in the linear-layer
        [out][in] layout: wq [Hq*d, dm], wk, wv [Hkv*d, dm], wo [dm, Hq*d],
        w_gate_up [2*d_ff, dm] (gate rows then up rows), w_down [dm, d_ff],
        and the gains g_attn, g_mlp [dm]; or the same through
        ``quantize_weights``.  ``kv_dtype``: the cache's, BF16, FP8_E4M3 or INT8."""
        self.w = list(weights)
        kinds = {isinstance(layer[name], tuple) for layer in self.w for name in PROJECTIONS}
        if len(kinds) != 1:
            raise ValueError("projections must all be bf16 tensors or all int8 codes with scales")
        if kv_dtype not in (N.BF16, N.FP8_E4M3, N.INT8):
            raise ValueError(f"kv_dtype {kv_dtype}: the layers' states are bf16")
        self.int8 = kinds.pop()
        self.hq, self.hkv, self.d, self.eps, self.theta = n_q_heads, n_kv_heads, head_dim, eps, theta
        wq, w_down = (w[0] if self.int8 else w for w in (self.w[0]["wq"], self.w[0]["w_down"]))
        self.d_model, self.d_ff = wq.shape[1], w_down.shape[1]
        self.pool = KVPool(len(self.w), n_q_heads, n_kv_heads, head_dim, n_blocks, max_seqs,
                           max_blocks_per_seq, kv_dtype, block_size, workspace_bytes=workspace_bytes)
        self._buf: Dict[str, torch.Tensor] = {}

    def _scratch_of(self, n: int) -> Dict[str, torch.Tensor]:
        """Scratch tensors of ``n`` tokens, by name."""
        bf, i8, f32 = torch.bfloat16, torch.int8, torch.float32
        want = {"q": (bf, n, self.hq, self.d), "k": (bf, n, self.hkv, self.d), "v": (bf, n, self.hkv, self.d),
                "o": (bf, n, self.hq * self.d), "gu": (bf, n, 2 * self.d_ff)}
        if self.int8:      # codes and scales of the left operands
            want.update(hq=(i8, n, self.d_model), oq=(i8, n, self.hq * self.d), aq=(i8, n, self.d_ff), s=(f32, n))
        else:
            want.update(h=(bf, n, self.d_model), a=(bf, n, self.d_ff))
        out = {}
        for name, (dtype, *shape) in want.items():
            size = 1
            for x in shape:
                size *= x
            t = self._buf.get(name)
            if t is None or t.numel() < size:
                t = self._buf[name] = torch.empty(size, dtype=dtype, device="cuda")
            out[name] = t[:size].view(*shape)
        return out

    def _run(self, fn, seq: int, x: torch.Tensor, pos0: int) -> torch.Tensor:
        n = x.shape[0]
        pos = torch.arange(pos0, pos0 + n, dtype=torch.int32, device="cuda")
        b = self._scratch_of(n)
        q, k, v, o, gu = (b[name] for name in ("q", "k", "v", "o", "gu"))
        x = x.clone()
        scale = self.d ** -0.5
        last = len(self.w) - 1
        for li, w in enumerate(self.w):
            qkv = (w["wq"], w["wk"], w["wv"])
            if self.int8:
                rows = rmsnorm_int8(x, w["g_attn"], self.eps, out=b["hq"], scales=b["s"])
                gemm_int8_multi(*rows, [c for c, _ in qkv], [s for _, s in qkv], (q, k, v))
            else:
                rmsnorm(x, w["g_attn"], self.eps, out=b["h"])
                gemm_bf16_multi(b["h"], qkv, (q, k, v))
            rope_qk_(q, k, pos, self.theta)
            rc = fn(li, [seq], [n], q, k, v, o, scale, commit=(li == last))
            if rc:
                raise N.PgsrError(rc, N.lib.pgsr_last_error().decode())
            if self.int8:
                gemm_int8(*quantize_rows(o, out=b["oq"], scales=b["s"]), *w["wo"], r=x, out=x)
                rows = rmsnorm_int8(x, w["g_mlp"], self.eps, out=b["hq"], scales=b["s"])
                gemm_int8(*rows, *w["w_gate_up"], out=gu)
                gemm_int8(*silu_mul_int8(gu, out=b["aq"], scales=b["s"]), *w["w_down"], r=x, out=x)
            else:
                gemm_bf16(o, w["wo"], r=x, out=x)                 # x <- x + O Wo
                rmsnorm(x, w["g_mlp"], self.eps, out=b["h"])
                gemm_silu_bf16(b["h"], w["w_gate_up"], gu, b["a"])
                gemm_bf16(b["a"], w["w_down"], r=x, out=x)        # x <- x + MLP(x)
        return x

    def replay(self, seq: int, x: torch.Tensor) -> torch.Tensor:
        """Tokens at positions len(seq) .. len(seq)+n-1 (Algorithm 1, replay loop)."""
        return self._run(self.pool.replay, seq, x, self.pool.seq_len(seq))

    def full_reset(self, seq: int, x: torch.Tensor) -> torch.Tensor:
        """Baseline B5: crop to 0 on the first layer, then all of x from position 0."""
        return self._run(self.pool.full_reset, seq, x, 0)

    def crop(self, seqs: List[int], new_lens: List[int]) -> int:
        return self.pool.crop(seqs, new_lens)

    def capture_restore_replay(self, seq: int, crop_len: int, x: torch.Tensor) -> "CapturedReplay":
        """Record the restore (crop of ``seq`` to ``crop_len``) and the replay
        of ``x`` through every layer as one HIP graph, from the pool state at
        this call.  Every library call of the two steps only enqueues kernels
        (no allocation, copy or memset on the stream), so the graph holds the
        launches the calls made, with the block ids the host mirror chose for
        that state.  Nothing runs during the capture: afterwards the host
        mirror reflects the recorded calls while the device is unchanged.
        Replaying is valid only from the captured state: restore it (device
        tables and host mirror, e.g. ``pool.load_meta``) before each replay."""
        n = x.shape[0]
        # scratch of its own, allocated before the capture and owned by the
        # result: the graph keeps these addresses, so eager calls that later
        # grow the shared scratch must not free them
        shared, self._buf = self._buf, {}
        try:
            self._scratch_of(n)
            xin = x.clone()
            stream = torch.cuda.Stream()
            stream.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.stream(stream):
                with torch.cuda.graph(graph, stream=stream):
                    rc = self.crop([seq], [crop_len])
                    if rc:
                        raise N.PgsrError(rc, N.lib.pgsr_last_error().decode())
                    out = self._run(self.pool.replay, seq, xin, crop_len)
            torch.cuda.current_stream().wait_stream(stream)
            own = self._buf
        finally:
            self._buf = shared
        return CapturedReplay(graph, xin, out, own)


class CapturedReplay:
    """A restore + replay recorded by DecoderReplay.capture_restore_replay:
    ``input`` holds the replayed token states (overwrite it in place to replay
    others), ``output`` receives the result of each ``replay()``."""

    def __init__(self, graph: "torch.cuda.CUDAGraph", inp: torch.Tensor, out: torch.Tensor,
                 scratch: Dict[str, torch.Tensor]):
        self.graph, self.input, self.output, self._scratch = graph, inp, out, scratch

    def replay(self) -> torch.Tensor:
        self.graph.replay()
        return self.output
