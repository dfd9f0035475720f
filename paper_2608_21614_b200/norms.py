"""The norms around a block with its gate and residual scale: plumbing over ``saem_block_norm``."""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B
from .mx import _allocated_on, _calls, _dtype

_GATES = {"none": B.SAEM_GATE_NONE, "token": B.SAEM_GATE_TOKEN, "channel": B.SAEM_GATE_CHANNEL, "full": B.SAEM_GATE_FULL}


class BlockNorm:
    """What stands between one block and the next on the residual stream x:

        z  = y / sqrt(mean(y^2) + eps) * w_post              (z = y without w_post)
        x' = residual_scale * x + branch_scale * g * z
        n  = x' / sqrt(mean(x'^2) + eps) * w_pre

    `gate`: "none" (g = 1), "token" [T] or [T, 1], "channel" [d] or [1, d], "full" [T, d]; with `gate_sigmoid`,
    g = 1 / (1 + exp(-gate))."""

    def __init__(self, d: int, w_post: Optional[torch.Tensor] = None, w_pre: Optional[torch.Tensor] = None, eps: float = 1e-6,
                 residual_scale: float = 1.0, branch_scale: float = 1.0, gate: str = "none", gate_sigmoid: bool = False):
        for w in (w_post, w_pre):
            if w is not None and (w.shape != (d,) or not w.is_contiguous()):
                raise B.SaemError(B.SAEM_ERR_SHAPE, "BlockNorm weight")
            if w is not None and not w.is_cuda:
                raise B.SaemError(B.SAEM_ERR_INVALID_ARG, "BlockNorm: weights on the GPU are wanted")
        if w_post is not None and w_pre is not None and (w_post.dtype, w_post.device) != (w_pre.dtype, w_pre.device):
            raise B.SaemError(B.SAEM_ERR_INVALID_ARG, "BlockNorm: weights of one type on one GPU are wanted")
        if gate not in _GATES:
            raise B.SaemError(B.SAEM_ERR_INVALID_ARG, "BlockNorm: gate %r" % (gate,))
        self.d, self.w_post, self.w_pre = d, w_post, w_pre
        w = w_post if w_post is not None else w_pre
        c = B.saem_norm_config(cols=d, w_dtype=B.SAEM_OUT_F32 if w is None else _dtype(w), gate_mode=_GATES[gate],
                               gate_sigmoid=int(gate_sigmoid), eps=eps, residual_scale=residual_scale, branch_scale=branch_scale)
        self._leave = bytes(c)              # rows, types and strides are the tensors'
        c.gate_mode = B.SAEM_GATE_NONE
        self._enter = bytes(c)

    def enter(self, x: torch.Tensor, n_out: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16,
              stream=None) -> torch.Tensor:
        """The first block's input: n of x itself."""
        if n_out is None:
            with _allocated_on(stream):
                n_out = torch.empty(x.shape[0], self.d, dtype=dtype, device=x.device)
        code = _calls.block_norm(self._enter, x, None, None, None, self.w_pre, None, n_out, stream)
        if code:
            raise B.SaemError(code, "BlockNorm")
        return n_out

    def leave(self, x: torch.Tensor, y: torch.Tensor, gate: Optional[torch.Tensor] = None, x_out: Optional[torch.Tensor] = None,
              n_out: Optional[torch.Tensor] = None, next_norm: bool = True, dtype: torch.dtype = torch.bfloat16, stream=None):
        """(x', n) after a block whose output is y; x_out (x's type) may be x.  `next_norm` False: x' only (n is None)."""
        if x_out is None:
            with _allocated_on(stream):
                x_out = torch.empty(x.shape[0], self.d, dtype=x.dtype, device=x.device)
        if n_out is None and next_norm:
            with _allocated_on(stream):
                n_out = torch.empty(x.shape[0], self.d, dtype=dtype, device=x.device)
        code = _calls.block_norm(self._leave, x, y, gate, self.w_post, self.w_pre if n_out is not None else None, x_out, n_out, stream)
        if code:
            raise B.SaemError(code, "BlockNorm")
        return x_out, n_out
