"""One transformer block's MoE half on 8-bit weights, from the library's calls:

    x1 = x + norm(attention output  W_o^T)      oled_norm_in, oled_fp8_matmul, oled_norm_out
    q  = norm(x1) in 8 bits                     oled_norm_in
    routes of the gate's logits q W_g^T         oled_fp8_matmul, oled_route_scored
    x  = x1 + norm(sum_j w_j expert_j(q))       oled_fp8_experts, oled_norm_out

A block owns its weights and its buffers (laid out once, for up to max_tokens), so
that a call makes eight library calls on one stream and nothing else, and can be
recorded in a HIP graph.

    python -m paper_2609_33385_amd.block8 --workload 3 --tokens 1 32 256
"""
from __future__ import annotations

import argparse
import concurrent.futures

import numpy as np
import torch

from . import harness
from . import oled
from . import workload as W


def quantise(w: torch.Tensor):
    """A weight matrix [N][K] (K a multiple of 128) in e4m3 with a scale per
    128 x 128, as oled_fp8_matmul takes its second operand."""
    N, K = w.shape
    nb = -(-N // 128)
    p = torch.zeros((nb * 128, K), dtype=torch.float32, device=w.device)
    p[:N] = w
    b = p.view(nb, 128, K // 128, 128)
    s = b.abs().amax((1, 3)).clamp_min(2.0 ** -100) / 448
    q = (b / s[:, None, :, None]).view(nb * 128, K)[:N].to(torch.float8_e4m3fn)
    return q.contiguous(), s.contiguous()


def pack_experts(w: W.Workload, seed: int, n_blocks: int, threads: int = 16) -> torch.Tensor:
    """[n_blocks][oled_fp8_expert_bytes] on the device: the workload's expert
    blocks 0 .. n_blocks - 1 in 8 bits."""
    out = np.zeros((n_blocks, oled.oled_fp8_expert_bytes(w.hidden, w.inter)), np.uint8)

    def one(b):
        w13, w2 = W.split_expert(w, W.expert_block(w, seed, b))
        oled.oled_fp8_pack_expert(w.dtype, w.hidden, w.inter, w13, w2, out[b])

    with concurrent.futures.ThreadPoolExecutor(max(1, min(threads, n_blocks))) as ex:
        list(ex.map(one, range(n_blocks)))
    return torch.from_numpy(out).cuda()


def _run(status: int, call: str) -> None:
    if status != oled.OLED_OK:
        raise oled.OledError(status, f"{call}: {oled.last_error(None)}")


def _check(t: torch.Tensor, what: str, dtype, least: int, device) -> None:
    """t holds at least `least` values of dtype (an int: of that many bytes), in order, on the device."""
    right = t.element_size() == dtype if isinstance(dtype, int) else t.dtype == dtype
    if not (right and t.numel() >= least and t.is_contiguous() and t.device == device):
        raise ValueError(f"{what} must be contiguous, on {device}, {least} values of "
                         f"{f'{dtype} byte' if isinstance(dtype, int) else dtype}: it is {tuple(t.shape)} of "
                         f"{t.dtype} on {t.device}")


class Block8:
    """forward(x, attn, ...) adds the block to x [T][H] bf16 in place. Only its last
    call writes x: where any call is refused, x is as it was.

    All calls of a block use its buffers. A forward on another stream than the last
    one's (the first: than the stream the block was made on) therefore waits for what
    that stream was given so far. Not while it is recorded in a graph: a caller orders
    the replays of a graph against other forwards of its block, and keeps the block
    while the graph is used."""

    def __init__(self, router: oled.Router, hidden: int, inter: int, max_tokens: int,
                 w_out, w_gate, experts: torch.Tensor, slot_of: torch.Tensor | None = None,
                 bias: torch.Tensor | None = None, norm_in: torch.Tensor | None = None,
                 norm_attn: torch.Tensor | None = None, norm_out: torch.Tensor | None = None,
                 eps: float = 1e-6):
        """w_out, w_gate: (e4m3, scales) of W_o [H][H] and the gate [E][H]
        (quantise); experts: packed blocks; slot_of [E] int32: the block of each
        expert (None: block e); bias [E] fp32: the router's balance bias; norm_*
        [H] fp32 (None for norm_attn and norm_out: that output has no norm). ValueError
        where a size is not one that the calls take or a tensor is too short for it."""
        E, k = router.n_experts, router.top_k
        self.router = oled.Router.from_buffer_copy(router)   # its logits are the block's own, in bf16
        self.hidden, self.inter, self.max_tokens = hidden, inter, max_tokens
        self.router.dtype = oled.DTYPES["bf16"]
        self.w_out, self.w_gate, self.experts, self.slot_of = w_out, w_gate, experts, slot_of
        self.bias, self.eps = bias, eps
        dev = experts.device
        self.norm_in = norm_in if norm_in is not None else torch.ones(hidden, device=dev)
        self.norm_attn, self.norm_out = norm_attn, norm_out
        if not 1 <= max_tokens <= 65535 or any(n % 128 or not 128 <= n <= 16384 for n in (hidden, inter)):
            raise ValueError("max_tokens must be in [1, 65535], hidden and inter multiples of 128 up to 16384")
        blocks = hidden // 128
        for w, what, rows in ((w_out, "w_out", hidden), (w_gate, "w_gate", E)):
            _check(w[0], what, 1, rows * hidden, dev)
            _check(w[1], f"{what}'s scales", torch.float32, -(-rows // 128) * blocks, dev)
        size = oled.oled_fp8_expert_bytes(hidden, inter)
        if experts.dim() != 2 or experts.shape[1] != size:
            raise ValueError(f"experts must be rows of {size} bytes: they are {tuple(experts.shape)}")
        _check(experts, "experts", 1, size * (1 if slot_of is not None else E), dev)
        for v, what, dtype, n in ((slot_of, "slot_of", torch.int32, E), (bias, "bias", torch.float32, E),
                                  (self.norm_in, "norm_in", torch.float32, hidden),
                                  (norm_attn, "norm_attn", torch.float32, hidden),
                                  (norm_out, "norm_out", torch.float32, hidden)):
            if v is not None:
                _check(v, what, dtype, n, dev)

        def ints(*n):
            return torch.empty(n, dtype=torch.int32, device=dev)

        # each call writes what the ones after it read
        T, routes = max_tokens, max_tokens * k
        self.q = torch.empty((T, hidden), dtype=torch.uint8, device=dev)
        self.q_scale = torch.empty((T, -(-hidden // 128)), dtype=torch.float32, device=dev)
        self.f = torch.empty((T, hidden), dtype=torch.bfloat16, device=dev)
        self.x1 = torch.empty((T, hidden), dtype=torch.bfloat16, device=dev)
        self.logits = torch.empty((T, E), dtype=torch.bfloat16, device=dev)
        self.topk_idx, self.weights = ints(T, k), torch.empty((T, k), device=dev)
        self.counts, self.offsets = ints(E), ints(E + 1)
        self.perm, self.inv_perm = ints(routes), ints(routes)
        self.routed = torch.empty((routes, hidden), dtype=torch.bfloat16, device=dev)
        self.route_ws = torch.empty(oled.oled_route_scored_workspace(T, E), dtype=torch.uint8,
                                    device=dev)
        self.expert_ws = torch.empty(oled.oled_fp8_experts_workspace(T, k, E, hidden, inter),
                                     dtype=torch.uint8, device=dev)
        self.last = torch.cuda.current_stream()   # of the last call
        self.streams = {self.last.cuda_stream}    # of all calls

    def _after_last(self, stream) -> None:
        """What `stream` is given from here on comes after the block's last call."""
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream)
        if stream.cuda_stream == self.last.cuda_stream:
            return
        with torch.cuda.stream(stream):
            if torch.cuda.is_current_stream_capturing():
                return
        stream.wait_event(self.last.record_event())
        if stream.cuda_stream not in self.streams:   # memory is given back after its work too
            for held in vars(self).values():
                for t in held if isinstance(held, tuple) else (held,):
                    if isinstance(t, torch.Tensor):
                        t.record_stream(stream)
            self.streams.add(stream.cuda_stream)
        self.last = stream

    def forward(self, x: torch.Tensor, attn: torch.Tensor, token_mask: torch.Tensor | None = None,
                gate: torch.Tensor | None = None, gate_tokens: int = 0, residual_scale: float = 1.0,
                stream=None) -> torch.Tensor:
        """x, attn [T][H] bf16, contiguous; token_mask [T] bool or bytes: tokens
        without routes where 0; gate: fp32 rows of H that scale the MoE output,
        token t under row t / gate_tokens (row 0 if gate_tokens is 0). ValueError where
        a tensor is of another type or too short."""
        T, H, k, E = x.shape[0], self.hidden, self.router.top_k, self.router.n_experts
        if not 1 <= T <= self.max_tokens or x.shape != (T, H) or attn.shape != (T, H):
            raise ValueError(f"x and attn must be [1..{self.max_tokens}][{H}]")
        if x.dtype != torch.bfloat16 or attn.dtype != torch.bfloat16 \
                or not (x.is_contiguous() and attn.is_contiguous()):
            raise ValueError("x and attn must be contiguous bf16")
        dev = self.experts.device
        if x.device != dev or attn.device != dev:
            raise ValueError(f"x and attn must be on {dev}")
        if token_mask is not None:
            _check(token_mask, "token_mask", 1, T, dev)
        if gate is not None:
            _check(gate, "gate", torch.float32, H * (-(-T // gate_tokens) if gate_tokens > 0 else 1), dev)
        s = stream if stream is not None else torch.cuda.current_stream()
        self._after_last(s)
        # the attention's output projection, onto the residual
        _run(oled.oled_norm_in(attn, "bf16", H, T, H, None, self.eps, None, self.q, self.q_scale, s),
             "oled_norm_in")
        _run(oled.oled_fp8_matmul(self.q, self.q_scale, H, *self.w_out, H, T, H, H, self.f, H, s),
             "oled_fp8_matmul")
        _run(oled.oled_norm_out(self.f, "bf16", None, None, 0, T, H, self.norm_attn, self.eps, None, 0,
                                x, residual_scale, self.x1, "bf16", s), "oled_norm_out")
        # the experts
        _run(oled.oled_norm_in(self.x1, "bf16", H, T, H, self.norm_in, self.eps, None, self.q, self.q_scale, s),
             "oled_norm_in")
        _run(oled.oled_fp8_matmul(self.q, self.q_scale, H, *self.w_gate, H, T, E, H, self.logits, E, s),
             "oled_fp8_matmul")
        _run(oled.oled_route_scored(self.router, self.logits, self.bias, token_mask, T, self.topk_idx,
                                    self.weights, self.counts, self.offsets, self.perm, self.inv_perm,
                                    None, self.route_ws, s), "oled_route_scored")
        _run(oled.oled_fp8_experts(self.q, self.q_scale, self.offsets, self.perm, T, k, E, H, self.inter,
                                   self.experts, self.experts.shape[0], self.slot_of, self.routed,
                                   self.expert_ws, s), "oled_fp8_experts")
        _run(oled.oled_norm_out(self.routed, "bf16", self.weights, self.inv_perm, k, T, H, self.norm_out,
                                self.eps, gate, gate_tokens, self.x1, residual_scale, x, "bf16", s),
             "oled_norm_out")
        return x


def make_block(w: W.Workload, seed: int, max_tokens: int, n_blocks: int | None = None,
               router: oled.Router | None = None, bias: torch.Tensor | None = None) -> Block8:
    """A block of the workload's shape. n_blocks < E: experts share blocks."""
    E, H = w.n_experts, w.hidden
    n = E if n_blocks is None else min(n_blocks, E)
    if router is None:
        router = oled.Router(n_experts=E, top_k=w.top_k, n_groups=8, top_groups=4, group_best=2,
                             score=oled.SCORES["sigmoid"], renorm=1, scale=1.0)
        if bias is None:
            bias = torch.zeros(E, device="cuda")
    slot_of = None if n == E else (torch.arange(E, dtype=torch.int32) % n).cuda()
    g = torch.Generator().manual_seed(seed)
    w_out = quantise((torch.randn((H, H), generator=g) / H ** 0.5).cuda())
    w_gate = quantise(harness.to_device(W.gate_weights(w, seed, 0)).float())
    # the gate's weights are drawn for activations of 0.02
    return Block8(router, H, w.inter, max_tokens, w_out, w_gate, pack_experts(w, seed, n), slot_of, bias,
                  norm_in=torch.full((H,), 0.02, device="cuda"),
                  norm_attn=torch.ones(H, device="cuda"), norm_out=torch.ones(H, device="cuda"))


def main() -> None:
    p = argparse.ArgumentParser(description="times the block, eager and as a graph")
    p.add_argument("--workload", type=int, default=3, choices=sorted(W.WORKLOADS))
    p.add_argument("--tokens", type=int, nargs="+", default=[1, 32, 256, 1024])
    p.add_argument("--blocks", type=int, default=16, help="expert blocks drawn (experts share them)")
    a = p.parse_args()
    w = W.WORKLOADS[a.workload]
    block = make_block(w, 0, max(a.tokens), a.blocks)
    for T in a.tokens:
        g = torch.Generator().manual_seed(T)
        attn = torch.randn((T, w.hidden), generator=g).bfloat16().cuda()
        x = torch.randn((T, w.hidden), generator=g).bfloat16().cuda()
        block.forward(x, attn)
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            block.forward(x, attn, stream=side)

        def us(call, n=50):
            call()
            start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            start.record()
            for _ in range(n):
                call()
            end.record()
            torch.cuda.synchronize()
            return 1e3 * start.elapsed_time(end) / n

        eager, replay = us(lambda: block.forward(x, attn)), us(graph.replay)
        print(f"{w.name}: {T} tokens, {eager:.1f} us a call, {replay:.1f} us a graph replay", flush=True)


if __name__ == "__main__":
    main()
