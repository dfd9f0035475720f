"""Rotary positions of heads, with the norm of each head in the same pass: plumbing over ``saem_rotate``."""
from __future__ import annotations

import math
from typing import List, Optional, Tuple

import torch

from . import binding as B
from .mx import _allocated_on, _calls


def frequencies(rotary_dim: int, base: float = 10000.0, scaling: Optional[dict] = None) -> Tuple[List[float], float]:
    """(radians per position of each pair, amplitude) in 64 bits.  Without `scaling` pair i turns by base^(-2i / rotary_dim).

    scaling["kind"], for contexts `factor` times as long as the model was trained for:
      "linear"  every pair turns `factor` times slower
      "base"    a larger base, so that the slowest pair turns `factor` times slower and the fastest as before
      "bands"   pairs with fewer than `low` turns within `original` positions turn `factor` times slower, those with more than `high`
                as before, and between them by a mean of the two, linear in the turns
      "yarn"    the same with the mean linear in the pair's index, between the pairs (rounded outwards) that turn beta_fast (32) and beta_slow (1) times, and
                sines and cosines multiplied by `amplitude` (0.1 ln factor + 1)"""
    n = rotary_dim // 2
    if rotary_dim < 0 or rotary_dim % 2 or not base > 0:
        raise B.SaemError(B.SAEM_ERR_INVALID_ARG, "frequencies: rotary_dim %r, base %r" % (rotary_dim, base))
    plain = [base ** (-2.0 * i / rotary_dim) for i in range(n)]
    if scaling is None:
        return plain, 1.0
    s = dict(scaling)
    try:
        kind, factor = s.pop("kind"), float(s.pop("factor"))
        if not (factor >= 1 and math.isfinite(factor)):
            raise ValueError("factor %r" % factor)
        if kind == "linear":
            result = [f / factor for f in plain], 1.0
        elif kind == "base":
            wider = base * factor ** (rotary_dim / (rotary_dim - 2)) if rotary_dim > 2 else base
            if not math.isfinite(wider):
                raise ValueError("base %r, factor %r" % (base, factor))
            result = [wider ** (-2.0 * i / rotary_dim) for i in range(n)], 1.0
        elif kind == "bands":
            original, low, high = float(s.pop("original")), float(s.pop("low")), float(s.pop("high"))
            if not (original > 0 and high > low):
                raise ValueError("original %r, low %r, high %r" % (original, low, high))
            keep = [min(1.0, max(0.0, (original * f / (2 * math.pi) - low) / (high - low))) for f in plain]
            result = [f * (k + (1 - k) / factor) for f, k in zip(plain, keep)], 1.0
        elif kind == "yarn":
            original, fast, slow = float(s.pop("original")), float(s.pop("beta_fast", 32.0)), float(s.pop("beta_slow", 1.0))
            amplitude = float(s.pop("amplitude", 0.1 * math.log(factor) + 1))
            if not (original > 0 and fast > slow > 0 and base > 1):
                raise ValueError("original %r, beta_fast %r, beta_slow %r" % (original, fast, slow))

            def index(turns):               # of the pair that turns so often within `original` positions
                return rotary_dim * math.log(original / (2 * math.pi * turns)) / (2 * math.log(base))
            first, last = max(0, math.floor(index(fast))), min(rotary_dim - 1, math.ceil(index(slow)))
            slower = [min(1.0, max(0.0, (i - first) / max(last - first, 0.001))) for i in range(n)]
            result = [f * ((1 - r) + r / factor) for f, r in zip(plain, slower)], amplitude
        else:
            raise ValueError("kind %r" % (kind,))
        if s:
            raise ValueError("unknown %s" % ", ".join(sorted(s)))
    except (KeyError, TypeError, ValueError, OverflowError) as e:
        raise B.SaemError(B.SAEM_ERR_INVALID_ARG, "frequencies: scaling: %s" % (e,)) from None
    return result


_PER_RADIAN = (10 ** 50 << 320) // (2 * 314159265358979323846264338327950288419716939937510)    # 2^320 / (2 pi)


def turns(radians: List[float]) -> List[int]:
    """Frequencies as fractions of a turn per position in units of 2^-64, as the kernels read them (signed 64-bit words)."""
    out = []
    for f in radians:
        n, d = f.as_integer_ratio()             # d is a power of two
        shift = 256 + d.bit_length() - 1
        u = (n * _PER_RADIAN + (1 << (shift - 1)) >> shift) % 2 ** 64
        out.append(u - 2 ** 64 if u >= 2 ** 63 else u)
    return out


class Rotary:
    """The rotation of a model's heads: the first `rotary_dim` elements (all, if not given; a multiple of 8) of heads of `head_dim`,
    pairs next to each other (`interleaved`) or half of `rotary_dim` apart.  `radians` (per position, with `amplitude`) in place of
    `base` and `scaling` (see `frequencies`)."""

    def __init__(self, head_dim: int, rotary_dim: Optional[int] = None, base: float = 10000.0, interleaved: bool = False,
                 scaling: Optional[dict] = None, radians: Optional[List[float]] = None, amplitude: float = 1.0, device="cuda"):
        rotary_dim = head_dim if rotary_dim is None else rotary_dim
        if head_dim < 8 or head_dim > 128 or head_dim % 8 or rotary_dim < 0 or rotary_dim > head_dim or rotary_dim % 8:
            raise B.SaemError(B.SAEM_ERR_SHAPE, "Rotary: head_dim %d, rotary_dim %d" % (head_dim, rotary_dim))
        if radians is None:
            radians, scale = frequencies(rotary_dim, base, scaling)
            amplitude *= scale
        if len(radians) != rotary_dim // 2:
            raise B.SaemError(B.SAEM_ERR_SHAPE, "Rotary: %d frequencies for %d pairs" % (len(radians), rotary_dim // 2))
        if not math.isfinite(amplitude) or not all(math.isfinite(f) for f in radians):
            raise B.SaemError(B.SAEM_ERR_INVALID_ARG, "Rotary: frequencies and amplitude have to be finite")
        self.head_dim, self.rotary_dim, self.interleaved, self.amplitude = head_dim, rotary_dim, bool(interleaved), float(amplitude)
        self.turns = torch.tensor(turns(radians), dtype=torch.int64, device=device)
        self._configs = {}

    def config(self, eps: float) -> B.saem_rotary_config:
        return B.saem_rotary_config(self.head_dim, self.rotary_dim, int(self.interleaved), eps, self.amplitude)

    def rotate(self, x: torch.Tensor, positions: torch.Tensor, weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
               out: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
        """x [tokens, heads, head_dim] at positions [tokens] (int32), each head normed and weighted first if `weight` [head_dim] is given.
        out: x itself, or heads of any type; without it new ones of `dtype` (x's)."""
        if out is None:
            with _allocated_on(stream):
                out = torch.empty(x.shape, dtype=dtype or x.dtype, device=x.device)
        c = self._configs.get(eps)
        if c is None:
            c = self._configs[eps] = bytes(B.saem_rotate_config(rotary=self.config(eps)))
        code = _calls.rotate(c, x, weight, self.turns, positions, out, stream)
        if code:
            raise B.SaemError(code, "rotate")
        return out
