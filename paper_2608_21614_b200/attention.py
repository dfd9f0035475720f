"""A paged cache of keys and values, appending to it, and attention over it: plumbing over ``saem_kv_append`` and ``saem_attend``.

As in `mx`, everything is enqueued on the current stream unless a stream is given, and nothing of a batch is read on the host, so
that calls can be captured and replayed while lengths, tables and offsets change."""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B
from .mx import _allocated_on, _calls
from .rotary import Rotary

_DTYPE = {torch.bfloat16: B.SAEM_OUT_BF16, torch.float16: B.SAEM_OUT_F16}


class PagedCache:
    """Keys and values of one layer: `k` and `v` [pages, kv_heads, page_size, head_dim], bfloat16 or float16; page_size a multiple of 16."""

    __slots__ = ("k", "v")

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        for t in (k, v):
            if not t.is_cuda or t.dim() != 4 or t.dtype not in _DTYPE or not t.is_contiguous() or t.data_ptr() % 16:
                raise B.SaemError(B.SAEM_ERR_INVALID_ARG, "PagedCache: [pages, kv_heads, page_size, head_dim] in bfloat16 or float16 on the GPU is wanted")
        if k.shape != v.shape or k.dtype != v.dtype or k.device != v.device:
            raise B.SaemError(B.SAEM_ERR_SHAPE, "PagedCache: keys and values have to be alike")
        pages, heads, page, dim = k.shape
        if pages < 1 or heads < 1 or heads > 65536 or page < 16 or page % 16 or page > 65536 or dim < 8 or dim % 8 or dim > 128 or pages * heads * page > 2 ** 31 - 1:
            raise B.SaemError(B.SAEM_ERR_SHAPE, "PagedCache: %s" % (tuple(k.shape),))
        self.k, self.v = k, v

    @classmethod
    def empty(cls, pages: int, kv_heads: int, page_size: int, head_dim: int, dtype: torch.dtype = torch.bfloat16, device="cuda") -> "PagedCache":
        """A cache whose contents are unspecified."""
        return cls(*(torch.empty(pages, kv_heads, page_size, head_dim, dtype=dtype, device=device) for _ in range(2)))

    @property
    def page_size(self) -> int:
        return self.k.shape[2]

    def nbytes(self) -> int:
        return 2 * self.k.numel() * self.k.element_size()


class Batch:
    """The sequences of a call, on the GPU: `offsets` [seqs + 1] (sequence s has the rows offsets[s] .. offsets[s + 1] - 1),
    `lengths` [seqs] (places in use, the new tokens included), `table` [seqs, pages of the longest] (all int32).  `max_new`: the most
    new tokens of a sequence; it chooses a kernel form, and a wrong one costs time and nothing else."""

    __slots__ = ("offsets", "lengths", "table", "max_new")

    def __init__(self, offsets: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor, max_new: int = 1):
        for t in (offsets, lengths, table):
            if not t.is_cuda or t.dtype != torch.int32 or t.device != table.device:
                raise B.SaemError(B.SAEM_ERR_INVALID_ARG, "Batch: int32 on one GPU is wanted")
        if lengths.dim() != 1 or offsets.shape != (lengths.shape[0] + 1,) or table.dim() != 2 or table.shape[0] < lengths.shape[0] or max_new < 0:
            raise B.SaemError(B.SAEM_ERR_SHAPE, "Batch")
        if not offsets.is_contiguous() or not lengths.is_contiguous() or (table.shape[1] > 1 and table.stride(1) != 1):
            raise B.SaemError(B.SAEM_ERR_INVALID_ARG, "Batch: consecutive entries are wanted")
        self.offsets, self.lengths, self.table, self.max_new = offsets, lengths, table, max_new


class Attention:
    """The attention of `q_heads` query heads over a cache.

    `append` norms (weights `w_q`, `w_k` [head_dim], float32 or bfloat16, where they are given) and rotates (`rotary`) new queries
    and keys; `attend` takes each token's softmax over the places up to its own (`causal`), of these the last `window` (0: all).
    Calls of one Attention must be ordered on the GPU (they share its workspace), and after the stream that was current when it was
    made; so must those of several with one workspace (`share`: the Attention whose workspace this one uses too, over a cache of the
    same head_dim at least)."""

    def __init__(self, q_heads: int, cache: PagedCache, rotary: Optional[Rotary] = None, w_q: Optional[torch.Tensor] = None,
                 w_k: Optional[torch.Tensor] = None, eps: float = 1e-6, scale: Optional[float] = None, causal: bool = True, window: int = 0,
                 share: Optional["Attention"] = None):
        pages, kv_heads, page, dim = cache.k.shape
        if q_heads < 1 or q_heads % kv_heads or q_heads // kv_heads > 128 or window < 0 or window > 2 ** 31 - 1:
            raise B.SaemError(B.SAEM_ERR_SHAPE, "Attention: %d query heads, %d key heads, window %d" % (q_heads, kv_heads, window))
        if rotary is not None and (rotary.head_dim != dim or rotary.turns.device != cache.k.device):
            raise B.SaemError(B.SAEM_ERR_SHAPE, "Attention: rotary of another head_dim or device")
        for w in (w_q, w_k):
            if w is not None and (w.shape != (dim,) or w.device != cache.k.device or w.dtype not in (torch.float32, torch.bfloat16)):
                raise B.SaemError(B.SAEM_ERR_SHAPE, "Attention: weights [head_dim] in float32 or bfloat16 beside the cache are wanted")
        self.q_heads, self.cache, self.rotary, self.w_q, self.w_k = q_heads, cache, rotary, w_q, w_k
        turn = rotary.config(eps) if rotary is not None else B.saem_rotary_config(dim, 0, 0, eps, 1.0)
        self._append = bytes(B.saem_append_config(rotary=turn, q_heads=q_heads))
        self._turns = rotary.turns if rotary is not None else None
        self._attend = bytes(B.saem_attend_config(q_heads=q_heads, causal=int(causal), window=window, scale=dim ** -0.5 if scale is None else scale))
        with torch.cuda.device(cache.k.device):
            size = B.saem_attend_workspace_bytes(B.saem_kv_cache(cache.k.data_ptr(), cache.v.data_ptr(), pages, page, kv_heads, dim, _DTYPE[cache.k.dtype]))
            if not size:
                raise B.SaemError(B.SAEM_ERR_CUDA, "Attention")
            if share is not None:
                if share.workspace.device != cache.k.device or share.workspace.numel() < size:
                    raise B.SaemError(B.SAEM_ERR_WORKSPACE, "Attention: the shared workspace is of another GPU or too small")
                self.workspace, self._status = share.workspace, share._status
                return
            raw = torch.empty(size + 1024, dtype=torch.uint8, device=cache.k.device)
            self.workspace = raw[-raw.data_ptr() % 1024:][:size]
            self.workspace[:B.SAEM_ATTEND_HEAD_BYTES].zero_()
        self._status = self.workspace[:4].view(torch.int32)

    def append(self, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, batch: Batch, positions: Optional[torch.Tensor] = None,
               q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
        """New q [tokens, q_heads, head_dim] (or None), k and v [tokens, kv_heads, head_dim], of one type: k and v into the cache, q to
        the result (the cache's type).  `positions` [tokens] int32: what is rotated by, in place of the places."""
        c = self.cache
        if q is not None and q_out is None:
            with _allocated_on(stream):
                q_out = torch.empty(q.shape, dtype=c.k.dtype, device=q.device)
        code = _calls.append(self._append, q, k, v, self.w_q, self.w_k, self._turns, positions, c.k, c.v, batch.offsets, batch.lengths,
                             batch.table, batch.max_new, q_out, self._status, stream)
        if code:
            raise B.SaemError(code, "append")
        return q_out

    def attend(self, q: torch.Tensor, batch: Batch, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
               stream=None) -> torch.Tensor:
        """q [tokens, q_heads, head_dim] (the cache's type) over the cache; lse [tokens, q_heads] float32, if given, becomes the logarithm of each
        row's sum of exponentials.  Rows behind the batch's last are left as they were; out must not be q."""
        if out is None:
            with _allocated_on(stream):
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        c = self.cache
        code = _calls.attend(self._attend, q, c.k, c.v, batch.offsets, batch.lengths, batch.table, batch.max_new, out, lse, self.workspace, stream)
        if code:
            raise B.SaemError(code, "attend")
        return out

    def device_status(self) -> int:
        """The status word of the calls so far, whatever their streams (synchronises the device): 0, SAEM_ERR_INVALID_ARG after a page
        outside the cache or a place outside the table, SAEM_ERR_TIMEOUT if a device-side wait ran out.  Clears it."""
        torch.cuda.synchronize(self.workspace.device)
        code = int(self._status.item())
        if code:                            # with the counters of a call that did not end
            self.workspace[:B.SAEM_ATTEND_HEAD_BYTES].zero_()
            torch.cuda.synchronize(self.workspace.device)
        return code
