"""The MoE half of a decoder with 4-bit experts: the operators of this package as a decoder uses them together.

Per layer, on a residual stream x (fp32) of T tokens:

    logits = n W_router^T                                        (saem_route_fused)
    y      = sum over the chosen experts of w_e FFN_e(n)         (saem_moe_step on MXFP4 experts)
    x, n   = x + g * rms(y) * w_post,  rms(x) * w_pre            (saem_block_norm; n is the next layer's input)

and behind the last layer a projection to the vocabulary with 4-bit weights (saem_mx_linear).  Attention is not part of
this package; a program with attention calls the same norm around it.

    python -m paper_2608_21614_b200.mx_block --layers 8 --tokens 1 --steps 64
"""
from __future__ import annotations

import argparse
import json
from typing import List, Optional, Sequence

import torch

from . import binding as B
from . import mx
from .layer import MoELayer
from .norms import BlockNorm


class MxMoEStack:
    """`n_layers` MoE layers over 4-bit experts with the norms between them, and a 4-bit head.

    Weights are given per layer: `experts[l]` a sequence of (gate, up, down) bf16 matrices on the GPU, `routers[l]`
    [E, d], `posts[l]`, `pres[l]` [d] (pres has one more entry, for the head's input), `head` [vocabulary, d]; all bf16."""

    def __init__(self, experts: Sequence[Sequence], routers: Sequence[torch.Tensor], posts: Sequence[torch.Tensor],
                 pres: Sequence[torch.Tensor], head: torch.Tensor, top_k: int, max_tokens: int, branch_scale: float = 1.0,
                 gate: Optional[Sequence[torch.Tensor]] = None):
        self.n_layers, E = len(experts), len(experts[0])
        f, d = experts[0][0][0].shape
        self.d, self.top_k, self.max_tokens = d, top_k, max_tokens
        for r in routers:                       # read by address
            if r.shape != (E, d) or r.dtype != torch.bfloat16 or not r.is_contiguous() or r.device != head.device or not r.is_cuda:
                raise B.SaemError(B.SAEM_ERR_INVALID_ARG, "MxMoEStack: routers [E, d] in bfloat16 on the GPU are wanted")
        self.layer = MoELayer(d, f, E, top_k, max_tokens, n_layers=self.n_layers, ffn_path=B.SAEM_FFN_MX)
        for l, layer in enumerate(experts):
            for e, matrices in enumerate(layer):
                self.layer.load_expert_mx(l, e, e, *(mx.quantize(m) for m in matrices))
        self.layer.copy_stream.synchronize()
        self.routers = list(routers)
        kind = "none" if gate is None else "channel"
        self.gates: List[Optional[torch.Tensor]] = [None] * self.n_layers if gate is None else list(gate)
        self.first = BlockNorm(d, w_pre=pres[0])
        self.norms = [BlockNorm(d, w_post=posts[l], w_pre=pres[l + 1], branch_scale=branch_scale, gate=kind) for l in range(self.n_layers)]
        self.head = mx.Linear(mx.quantize(head), max_tokens)
        dev = head.device
        self.n = torch.empty(max_tokens, d, dtype=torch.bfloat16, device=dev)
        self.y = torch.empty(max_tokens, d, dtype=torch.float32, device=dev)
        self.logits = torch.empty(max_tokens, E, dtype=torch.float32, device=dev)
        self.vocabulary = torch.empty(max_tokens, head.shape[0], dtype=torch.float32, device=dev)

    def block(self, l: int, x: torch.Tensor) -> torch.Tensor:
        """Layer l on the residual stream x [T, d] fp32, in place; self.n holds the layer's input and then the next one's."""
        T, h = x.shape[0], self.layer.ctx.handle
        n, y, logits = self.n[:T], self.y[:T], self.logits[:T]
        B.saem_route_fused(h, n, self.routers[l], T, logits, self.layer.topk_idx, self.layer.topk_w)
        B.saem_moe_step(h, None, l, logits, n, T, y)
        self.norms[l].leave(x, y, gate=self.gates[l], x_out=x, n_out=n)
        return x

    def step(self, x: torch.Tensor) -> torch.Tensor:
        """All layers on x [T, d] fp32 (in place); the head's logits [T, vocabulary] fp32."""
        T = x.shape[0]
        self.first.enter(x, n_out=self.n[:T])
        for l in range(self.n_layers):
            self.block(l, x)
        return self.head(self.n[:T], out=self.vocabulary[:T])

    def capture(self, x: torch.Tensor) -> torch.cuda.CUDAGraph:
        """One step on x as a CUDA graph; its logits are self.vocabulary[:T]."""
        keep = x.clone()
        side = torch.cuda.Stream(device=x.device)
        side.wait_stream(torch.cuda.current_stream(x.device))
        with torch.cuda.stream(side):
            self.step(x)                        # first calls outside the capture
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                self.step(x)
        torch.cuda.current_stream(x.device).wait_stream(side)
        x.copy_(keep)
        return graph

    def device_status(self) -> int:
        return self.layer.device_status() or self.head.device_status()

    def close(self):
        self.layer.close()


def random_stack(d: int, f: int, E: int, top_k: int, n_layers: int, vocabulary: int, max_tokens: int, seed: int = 0, **kw) -> MxMoEStack:
    """A stack with random weights of the usual scale."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def r(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(torch.bfloat16)
    experts = [[(r(f, d, scale=d ** -0.5), r(f, d, scale=d ** -0.5), r(d, f, scale=f ** -0.5)) for _ in range(E)] for _ in range(n_layers)]
    ones = lambda: 1 + 0.1 * r(d)                                               # noqa: E731
    return MxMoEStack(experts, [r(E, d, scale=d ** -0.5) for _ in range(n_layers)], [ones() for _ in range(n_layers)],
                      [ones() for _ in range(n_layers + 1)], r(vocabulary, d, scale=d ** -0.5), top_k, max_tokens, **kw)


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--layers", type=int, default=8)
    p.add_argument("--tokens", type=int, default=1)
    p.add_argument("--steps", type=int, default=64)
    p.add_argument("--d-model", type=int, default=2048)
    p.add_argument("--d-ff", type=int, default=768)
    p.add_argument("--experts", type=int, default=128)
    p.add_argument("--top-k", type=int, default=8)
    p.add_argument("--vocabulary", type=int, default=32768)
    a = p.parse_args()
    stack = random_stack(a.d_model, a.d_ff, a.experts, a.top_k, a.layers, a.vocabulary, a.tokens)
    x = torch.randn(a.tokens, a.d_model, device="cuda")
    graph = stack.capture(x)
    for _ in range(3):
        graph.replay()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(a.steps):
        graph.replay()
    end.record()
    end.synchronize()
    assert stack.device_status() == 0
    slot = stack.layer.ctx.slot_bytes
    print(json.dumps({"ms_per_step": round(begin.elapsed_time(end) / a.steps, 4), "layers": a.layers, "tokens": a.tokens,
                      "slot_bytes": slot, "bf16_slot_bytes": 6 * a.d_model * a.d_ff, "data": "synthetic"}))
    stack.close()


if __name__ == "__main__":
    main()
