"""A decoder with 4-bit experts, or the MoE half of one: the operators of this package as a decoder uses them together.

Per layer, on a residual stream x (fp32) of T tokens, where the layers have attention:

    q k v  = n W_qkv^T                                           (saem_mx_linear)
    q      = rotated rms(q) * w_q;  k likewise and v to the cache  (saem_kv_append)
    y      = softmax(q k^T) v over the cache, then W_out         (saem_attend, saem_mx_linear)
    x, n   = x + rms(y) * w_post,  rms(x) * w_pre                (saem_block_norm)

and always:

    logits = n W_router^T                                        (saem_route_fused)
    y      = sum over the chosen experts of w_e FFN_e(n)         (saem_moe_step on MXFP4 experts)
    x, n   = x + g * rms(y) * w_post,  rms(x) * w_pre            (saem_block_norm; n is the next layer's input)

and behind the last layer a projection to the vocabulary with 4-bit weights (saem_mx_linear).  Without attention a program
calls its own and the same norm around it.

    python -m paper_2608_21614_b200.mx_block --layers 8 --tokens 1 --steps 64 [--context 4096]
"""
from __future__ import annotations

import argparse
import json
from typing import List, Optional, Sequence

import torch

from . import binding as B
from . import mx
from .attention import Attention, Batch, PagedCache
from .layer import MoELayer
from .norms import BlockNorm
from .rotary import Rotary


def _first_status(parts) -> int:
    """The first status that is set, all of them read and cleared."""
    return next(filter(None, [p.device_status() for p in parts]), 0)


class MxAttention:
    """The attention half of a layer, its projections in 4 bits.

    `w_qkv` [(q_heads + 2 kv_heads) * head_dim, d] (queries, keys, values) and `w_out` [d, q_heads * head_dim] bf16 on the GPU; `post` and `pre` [d]
    the norms behind it (post may be None); the other arguments are Attention's.  `share`: another layer's MxAttention, whose
    attention workspace and buffers this one uses too (layers run one after the other).

    Rows behind the batch's last sequence (spare ones of a captured step) are not attended: what the buffers held there, zeros or an
    earlier call's, is projected and added to them, so that their x and n have no meaning.  No other row depends on them, whatever they hold."""

    def __init__(self, w_qkv: torch.Tensor, w_out: torch.Tensor, post: Optional[torch.Tensor], pre: torch.Tensor, cache: PagedCache, q_heads: int,
                 max_tokens: int, rotary: Optional[Rotary] = None, w_q: Optional[torch.Tensor] = None, w_k: Optional[torch.Tensor] = None,
                 window: int = 0, branch_scale: float = 1.0, share: Optional["MxAttention"] = None):
        _, kv_heads, _, dim = cache.k.shape
        self.heads, self.d, self.max_tokens = (q_heads, kv_heads, dim), w_out.shape[0], max_tokens
        if w_qkv.shape != ((q_heads + 2 * kv_heads) * dim, self.d) or w_out.shape != (self.d, q_heads * dim):
            raise B.SaemError(B.SAEM_ERR_SHAPE, "MxAttention: projections")
        if cache.k.dtype != torch.bfloat16:                                         # the projection behind it takes no other 16-bit type
            raise B.SaemError(B.SAEM_ERR_INVALID_ARG, "MxAttention: a cache in bfloat16 is wanted")
        if share is not None and (share.heads, share.d, share.max_tokens) != (self.heads, self.d, max_tokens):
            raise B.SaemError(B.SAEM_ERR_SHAPE, "MxAttention: buffers of another layer shape")
        self.qkv, self.out = mx.Linear(mx.quantize(w_qkv), max_tokens), mx.Linear(mx.quantize(w_out), max_tokens)
        self.attention = Attention(q_heads, cache, rotary=rotary, w_q=w_q, w_k=w_k, window=window, share=share.attention if share is not None else None)
        self.norm = BlockNorm(self.d, w_post=post, w_pre=pre, branch_scale=branch_scale)
        if share is not None:
            self.projected, self.rotated, self.weighted, self.y = share.projected, share.rotated, share.weighted, share.y
            return
        dev = cache.k.device
        self.projected = torch.zeros(max_tokens, q_heads + 2 * kv_heads, dim, dtype=torch.bfloat16, device=dev)
        self.rotated, self.weighted = (torch.zeros(max_tokens, q_heads, dim, dtype=cache.k.dtype, device=dev) for _ in range(2))
        self.y = torch.empty(max_tokens, self.d, dtype=torch.float32, device=dev)

    def __call__(self, x: torch.Tensor, n: torch.Tensor, batch: Batch) -> None:
        """x [T, d] fp32 and its normed form n [T, d] bf16, both in place: n becomes the input of the layer's other half."""
        T, (hq, hk, _) = x.shape[0], self.heads
        qkv, q, a, y = self.projected[:T], self.rotated[:T], self.weighted[:T], self.y[:T]
        self.qkv(n, out=qkv.flatten(1))
        self.attention.append(qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:], batch, q_out=q)
        self.attention.attend(q, batch, out=a)
        self.out(a.flatten(1), out=y)
        self.norm.leave(x, y, x_out=x, n_out=n)

    def device_status(self) -> int:
        return _first_status((self.qkv, self.attention, self.out))


class MxMoEStack:
    """`n_layers` MoE layers over 4-bit experts with the norms between them, and a 4-bit head.

    `attention`: an MxAttention for each layer, run before its experts (`pres[l]` are then the norms before attention, and a step
    takes the Batch of its tokens; results of rows behind the batch's last sequence have no meaning).

    Weights are given per layer: `experts[l]` a sequence of (gate, up, down) bf16 matrices on the GPU, `routers[l]`
    [E, d], `posts[l]`, `pres[l]` [d] (pres has one more entry, for the head's input), `head` [vocabulary, d]; all bf16."""

    def __init__(self, experts: Sequence[Sequence], routers: Sequence[torch.Tensor], posts: Sequence[torch.Tensor],
                 pres: Sequence[torch.Tensor], head: torch.Tensor, top_k: int, max_tokens: int, branch_scale: float = 1.0,
                 gate: Optional[Sequence[torch.Tensor]] = None, attention: Optional[Sequence[MxAttention]] = None):
        self.n_layers, E = len(experts), len(experts[0])
        f, d = experts[0][0][0].shape
        self.d, self.top_k, self.max_tokens = d, top_k, max_tokens
        for r in routers:                       # read by address
            if r.shape != (E, d) or r.dtype != torch.bfloat16 or not r.is_contiguous() or r.device != head.device or not r.is_cuda:
                raise B.SaemError(B.SAEM_ERR_INVALID_ARG, "MxMoEStack: routers [E, d] in bfloat16 on the GPU are wanted")
        self.attention = None if attention is None else list(attention)
        if self.attention is not None and (len(self.attention) != self.n_layers or any(a.d != d or a.max_tokens < max_tokens for a in self.attention)):
            raise B.SaemError(B.SAEM_ERR_SHAPE, "MxMoEStack: an MxAttention of the layers' width for each of them is wanted")
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

    def block(self, l: int, x: torch.Tensor, batch: Optional[Batch] = None) -> torch.Tensor:
        """Layer l on the residual stream x [T, d] fp32, in place; self.n holds the layer's input and then the next one's."""
        T, h = x.shape[0], self.layer.ctx.handle
        n, y, logits = self.n[:T], self.y[:T], self.logits[:T]
        if self.attention is not None:
            if batch is None:
                raise B.SaemError(B.SAEM_ERR_INVALID_ARG, "MxMoEStack: layers with attention take the Batch of their tokens")
            self.attention[l](x, n, batch)
        B.saem_route_fused(h, n, self.routers[l], T, logits, self.layer.topk_idx, self.layer.topk_w)
        B.saem_moe_step(h, None, l, logits, n, T, y)
        self.norms[l].leave(x, y, gate=self.gates[l], x_out=x, n_out=n)
        return x

    def step(self, x: torch.Tensor, batch: Optional[Batch] = None) -> torch.Tensor:
        """All layers on x [T, d] fp32 (in place); the head's logits [T, vocabulary] fp32."""
        T = x.shape[0]
        self.first.enter(x, n_out=self.n[:T])
        for l in range(self.n_layers):
            self.block(l, x, batch)
        return self.head(self.n[:T], out=self.vocabulary[:T])

    def capture(self, x: torch.Tensor, batch: Optional[Batch] = None) -> torch.cuda.CUDAGraph:
        """One step on x as a CUDA graph; its logits are self.vocabulary[:T].  The batch's tensors are read anew by every replay."""
        keep = x.clone()
        side = torch.cuda.Stream(device=x.device)
        side.wait_stream(torch.cuda.current_stream(x.device))
        with torch.cuda.stream(side):
            self.step(x, batch)                 # first calls outside the capture
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                self.step(x, batch)
        torch.cuda.current_stream(x.device).wait_stream(side)
        x.copy_(keep)
        return graph

    def device_status(self) -> int:
        return _first_status((self.layer, self.head, *(self.attention or ())))

    def close(self):
        self.layer.close()


def random_stack(d: int, f: int, E: int, top_k: int, n_layers: int, vocabulary: int, max_tokens: int, seed: int = 0, heads=None, pages: int = 0,
                 page_size: int = 64, **kw) -> MxMoEStack:
    """A stack with random weights of the usual scale; heads: (query heads, key heads, head_dim) of layers with attention, whose
    caches have `pages` pages each."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def r(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(torch.bfloat16)
    experts = [[(r(f, d, scale=d ** -0.5), r(f, d, scale=d ** -0.5), r(d, f, scale=f ** -0.5)) for _ in range(E)] for _ in range(n_layers)]
    ones = lambda n=d: 1 + 0.1 * r(n)                                           # noqa: E731
    if heads is not None:
        hq, hk, dim = heads
        turn, layers = Rotary(dim), []
        for _ in range(n_layers):
            layers.append(MxAttention(r((hq + 2 * hk) * dim, d, scale=d ** -0.5), r(d, hq * dim, scale=(hq * dim) ** -0.5), ones(), ones(),
                                      PagedCache.empty(pages, hk, page_size, dim), hq, max_tokens, rotary=turn, w_q=ones(dim), w_k=ones(dim),
                                      share=layers[0] if layers else None))
        kw["attention"] = layers
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
    p.add_argument("--context", type=int, default=0, help="places of each sequence before the first step; 0: layers without attention")
    p.add_argument("--q-heads", type=int, default=32)
    p.add_argument("--kv-heads", type=int, default=4)
    p.add_argument("--head-dim", type=int, default=128)
    p.add_argument("--page-size", type=int, default=64)
    a = p.parse_args()
    batch, kw = None, {}
    if a.context:                               # one new token of each sequence, a step after the other
        per = -(-(a.context + a.steps + 4) // a.page_size)
        kw = {"heads": (a.q_heads, a.kv_heads, a.head_dim), "pages": per * a.tokens, "page_size": a.page_size}
        batch = Batch(torch.arange(a.tokens + 1, dtype=torch.int32, device="cuda"), torch.full((a.tokens,), a.context + 1, dtype=torch.int32, device="cuda"),
                      torch.randperm(per * a.tokens, device="cuda").to(torch.int32).view(a.tokens, per))
    stack = random_stack(a.d_model, a.d_ff, a.experts, a.top_k, a.layers, a.vocabulary, a.tokens, **kw)
    for layer in stack.attention or ():         # what a prompt would have left there
        layer.attention.cache.k.normal_()
        layer.attention.cache.v.normal_()
    x = torch.randn(a.tokens, a.d_model, device="cuda")
    graph = stack.capture(x, batch)

    def step():
        graph.replay()
        if batch is not None:
            batch.lengths.add_(1)
    for _ in range(3):
        step()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(a.steps):
        step()
    end.record()
    end.synchronize()
    assert stack.device_status() == 0
    slot = stack.layer.ctx.slot_bytes
    print(json.dumps({"ms_per_step": round(begin.elapsed_time(end) / a.steps, 4), "layers": a.layers, "tokens": a.tokens, "context": a.context,
                      "slot_bytes": slot, "bf16_slot_bytes": 6 * a.d_model * a.d_ff, "data": "synthetic"}))
    stack.close()


if __name__ == "__main__":
    main()
