"""The attention operators in 64 bits, one token and head at a time or in rows, for the tests."""
import math

import torch


def rotation(x, positions, radians, interleaved=False, amplitude=1.0, w=None, eps=1e-6):
    """x [T, heads, dim] float64; the first 2 * len(radians) elements of each head turn."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    n = len(radians)
    angle = positions.double()[:, None] * torch.tensor(radians, dtype=torch.float64, device=x.device)
    c, s = (amplitude * torch.cos(angle))[:, None], (amplitude * torch.sin(angle))[:, None]
    out = x.clone()
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if interleaved else (x[..., :n], x[..., n:2 * n])
    ya, yb = a * c - b * s, b * c + a * s
    if interleaved:
        out[..., 0:2 * n:2], out[..., 1:2 * n:2] = ya, yb
    else:
        out[..., :n], out[..., n:2 * n] = ya, yb
    return out


def gather(cache, table, length, page):
    """[kv_heads, length, dim] of one sequence, in its own type."""
    if length == 0:
        return cache[:0, :, 0].transpose(0, 1)
    pages = table[:-(-length // page)].long()
    return cache[pages].transpose(0, 1).flatten(1, 2)[:, :length]


def attend(q, k, v, n, causal, window, scale):
    """q [n, q_heads, dim] of one sequence's last n places, k, v [kv_heads, len, dim]: (out, size, lse, spread) in float64, where size is
    sum_j p_j |v_j| and spread the largest scale * sum |q| |k_j| of a row.  What a row does not see is not touched."""
    q, k, v = q.double(), k.double(), v.double()
    heads, length, dim = q.shape[1], k.shape[1], q.shape[2]
    group = heads // k.shape[0]
    out, size = torch.zeros_like(q), torch.zeros_like(q)
    lse, spread = torch.full((n, heads), -math.inf, dtype=torch.float64, device=q.device), torch.zeros(n, heads, dtype=torch.float64, device=q.device)
    place = length - n + torch.arange(n, device=q.device)
    j = torch.arange(length, device=q.device)
    seen = torch.ones(n, length, dtype=torch.bool, device=q.device)
    if causal:
        seen &= j <= place[:, None]
    if window:
        seen &= j > place[:, None] - window
    some = seen.any(1)
    if not some.any():
        return out, size, lse, spread
    for h in range(heads):
        kh, vh = k[h // group], v[h // group]
        s = torch.where(seen, scale * (q[:, h] @ torch.nan_to_num(kh, 0.0, 0.0, 0.0).T), -math.inf)
        for t in torch.nonzero(~torch.isfinite(kh).all(1)).flatten().tolist():          # keys that are not finite: rows that see them
            s[:, t] = torch.where(seen[:, t], scale * (q[:, h] @ kh[t]), -math.inf)
        p = torch.softmax(torch.where(some[:, None], s, 0.0), 1) * some[:, None]
        whole = torch.nan_to_num(vh, 0.0, 0.0, 0.0)
        out[:, h], size[:, h] = p @ whole, p @ whole.abs()
        for t in torch.nonzero(~torch.isfinite(vh).all(1)).flatten().tolist():
            extra = (p[:, t, None] * vh[t]) * seen[:, t, None]
            out[:, h] = torch.where(seen[:, t, None], out[:, h] + extra - p[:, t, None] * whole[t], out[:, h])
        lse[:, h] = torch.where(some, torch.logsumexp(s, 1), -math.inf)
        spread[:, h] = torch.where(seen, scale * (q[:, h].abs() @ torch.nan_to_num(kh, 0.0, 0.0, 0.0).abs().T), 0.0).amax(1)
    return out, size, lse, spread
