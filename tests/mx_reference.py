"""Plain 64-bit implementations of the microscaled 4-bit operators and of the block norms, for the tests."""
import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(x):
    """(values, codes, scale bytes) of x [rows, cols]: every element to the nearest of the eight magnitudes, ties to the
    even code; values and codes padded with zeros to whole blocks."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    pad = -cols % 32
    v = np.pad(x, ((0, 0), (0, pad))).reshape(rows, -1, 32)
    amax = np.abs(v).max(-1)
    finite = np.isfinite(amax)
    exponent = np.frexp(np.where(finite & (amax > 0), amax, 2.0 ** -140))[1] - 1          # floor(log2)
    s = np.where(finite, np.maximum(exponent - 2, -127) + 127, 255).astype(np.int64)
    scale = np.where(finite, np.ldexp(1.0, s - 127), np.nan)
    a = np.abs(v) / np.where(finite, scale, 1.0)[..., None]
    distance = np.abs(np.where(np.isfinite(a), a, 0.0)[..., None] - E2M1)
    best = distance.min(-1, keepdims=True)
    hit = distance == best
    even = hit & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), hit.argmax(-1))
    code = np.where(finite[..., None], code, 0)
    sign = np.signbit(v) & finite[..., None]
    values = np.where(sign, -1.0, 1.0) * E2M1[code] * scale[..., None]
    return values.reshape(rows, -1)[:, :cols], (code | sign.astype(np.int64) << 3).reshape(rows, -1), s


def pack_codes(codes):
    return (codes[:, 0::2] | codes[:, 1::2] << 4).astype(np.uint8)


def scale_at(rows, n_block):
    """Byte offset of the scale of (row, block) in the tiled scale array."""
    r, b = np.meshgrid(np.arange(rows), np.arange(n_block), indexing="ij")
    n_span = (n_block + 3) // 4
    return ((r // 128) * n_span + b // 4) * 512 + (r % 32) * 16 + (r // 32 % 4) * 4 + b % 4


def silu(z):
    return z / (1 + np.exp(-z))


def moe(x, idx, w, gate, up, down, n_shared=0):
    """(out, bound): out[t] = sum_j w[t, j] y_j (+ shared) from dequantised matrices in 64 bits, and with it the sum of
    the magnitudes |w_j| |Wd| |h| that rounding errors of h are proportional to."""
    T, d = x.shape
    E = len(gate) - n_shared
    out, bound = np.zeros((T, d)), np.zeros((T, d))
    for t in range(T):
        pairs = [(int(e), float(v)) for e, v in zip(idx[t], w[t])] + [(E + s, 1.0) for s in range(n_shared)]
        for e, v in pairs:
            h = silu(gate[e] @ x[t]) * (up[e] @ x[t])
            out[t] += v * (down[e] @ h)
            bound[t] += abs(v) * (np.abs(down[e]) @ np.abs(h))
    return out, bound


def block_norm(x, y=None, gate=None, sigmoid=False, w_post=None, w_pre=None, eps=1e-6, a=1.0, b=1.0):
    """(x', n, magnitude of x''s terms)."""
    x = np.asarray(x, np.float64)
    size = np.abs(x)
    if y is not None:
        z = np.asarray(y, np.float64)
        if w_post is not None:
            z = z / np.sqrt((z * z).mean(-1, keepdims=True) + eps) * w_post
        if gate is not None:
            g = np.asarray(gate, np.float64)
            z = z * (1 / (1 + np.exp(-g)) if sigmoid else g)
        size = np.abs(a * x) + np.abs(b * z)
        x = a * x + b * z
    n = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x, n if w_pre is None else n * w_pre, size
