"""The block norms against the formula in 64 bits.  fp32 arithmetic: each of x''s terms carries a handful of roundings
(a sum of up to 16384 squares in a tree, a root, a division, four products): 2^-20 of their magnitudes covers them; a bf16
output rounds once more, by half a unit of 8 significant bits: 2^-8 of its value."""
import numpy as np
import pytest
import torch

import mx_reference as ref

pytestmark = pytest.mark.gpu
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def f64(t):
    return None if t is None else t.detach().float().cpu().numpy().astype(np.float64)


def check(norm, x, y, gate=None, sigmoid=False, eps=1e-6, a=1.0, b=1.0, n_dtype="bf16", x_out=None, n_out=None):
    want_x, want_n, size = ref.block_norm(f64(x), f64(y), f64(gate), sigmoid, f64(norm.w_post), f64(norm.w_pre), eps, a, b)
    got_x, got_n = norm.leave(x, y, gate=gate, x_out=x_out, n_out=n_out, dtype=TORCH[n_dtype])
    limit = 2.0 ** -20 * size
    if got_x.dtype == torch.bfloat16:
        limit = limit + 2.0 ** -8 * 1.01 * np.abs(want_x)
    assert (np.abs(f64(got_x) - want_x) <= limit).all()
    per = np.sqrt((want_x ** 2).mean(-1, keepdims=True) + eps)
    w = 1.0 if norm.w_pre is None else np.abs(f64(norm.w_pre))
    limit = 2.0 ** -20 * (size / per * w + np.abs(want_n))
    if got_n.dtype == torch.bfloat16:
        limit = limit + 2.0 ** -8 * 1.01 * np.abs(want_n)
    assert (np.abs(f64(got_n) - want_n) <= limit).all()
    return got_x, got_n


def data(T, d, x="bf16", y="f32", seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + T * 131 + d)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")                         # noqa: E731
    return ((3 * r(T, d)).to(TORCH[x]), (0.3 * r(T, d)).to(TORCH[y]), (1 + 0.1 * r(d)), (1 + 0.1 * r(d)), r)


@pytest.mark.parametrize("x,y,w", [("bf16", "f32", "bf16"), ("f32", "bf16", "f32"), ("bf16", "bf16", "bf16"), ("f32", "f32", "bf16")])
@pytest.mark.parametrize("T,d", [(1, 1), (1, 2048), (2, 7), (3, 64), (5, 65), (2, 248), (9, 513), (33, 1000), (4, 2560), (7, 4096),
                                 (3, 4097), (2, 8200), (2, 16384), (2, 16383), (700, 128)])
def test_leave(T, d, x, y, w):
    from paper_2608_21614_b200.norms import BlockNorm
    xs, ys, w_post, w_pre, _ = data(T, d, x, y)
    norm = BlockNorm(d, w_post.to(TORCH[w]), w_pre.to(TORCH[w]), residual_scale=0.75, branch_scale=-1.25)
    check(norm, xs, ys, a=0.75, b=-1.25, n_dtype="f32" if x == "f32" else "bf16")


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("gate", ["token", "channel", "full"])
@pytest.mark.parametrize("T,d", [(1, 128), (6, 200), (5, 129), (3, 2048)])
def test_gates(T, d, gate, sigmoid):
    from paper_2608_21614_b200.norms import BlockNorm
    xs, ys, w_post, w_pre, r = data(T, d)
    for dtype in TORCH.values():
        g = (4 * r(*{"token": (T, 1), "channel": (1, d), "full": (T, d)}[gate])).to(dtype)
        for post in (w_post, None):
            check(BlockNorm(d, post, w_pre, gate=gate, gate_sigmoid=sigmoid), xs, ys, gate=g, sigmoid=sigmoid)
    check(BlockNorm(d, w_post, None, gate=gate), xs, ys, gate=r(*g.shape))


def test_strides_in_place_and_single_outputs():
    from paper_2608_21614_b200.norms import BlockNorm
    xs, ys, w_post, w_pre, r = data(6, 96, "f32", "bf16")
    norm = BlockNorm(96, w_post, w_pre)
    want_x, want_n = check(norm, xs, ys)
    for pad, off in ((8, 8), (3, 1)):                                                    # aligned rows and unaligned ones
        wide = lambda t: torch.zeros(6, 96 + pad, dtype=t.dtype, device="cuda")[:, off:off + 96].copy_(t)   # noqa: E731
        a, b, n = wide(xs), wide(ys), torch.full((6, 96 + pad), 9.0, device="cuda").to(torch.bfloat16)
        check(norm, a, b, n_out=n[:, off:off + 96])
        assert (n[:, :off] == 9).all() and (n[:, off + 96:] == 9).all()
    x2 = xs.clone()
    got_x, got_n = norm.leave(x2, ys, x_out=x2)
    assert got_x is x2 and torch.equal(x2, want_x) and torch.equal(got_n, want_n)
    only_x, none = norm.leave(xs, ys, next_norm=False)
    assert none is None and torch.equal(only_x, want_x)
    token = BlockNorm(96, w_post, w_pre, gate="token")
    g = r(6, 5)[:, 2]                                                                    # one value per token, five apart
    check(token, xs, ys, gate=g[:, None])
    n = norm.enter(xs)
    _, want, size = ref.block_norm(f64(xs), w_pre=f64(w_pre))
    assert (np.abs(f64(n) - want) <= 2.0 ** -8 * np.abs(want) + 1e-6).all()
    assert norm.enter(xs[:0]).shape == (0, 96)


@pytest.mark.parametrize("scale", [0.0, 1e-25, 1e15])
def test_extreme_rows(scale):
    from paper_2608_21614_b200.norms import BlockNorm
    xs, ys, w_post, w_pre, _ = data(4, 256, "f32", "f32")
    check(BlockNorm(256, w_post, w_pre), xs * scale, ys * scale)


def test_a_row_that_is_not_finite_stays_alone():
    from paper_2608_21614_b200.norms import BlockNorm
    xs, ys, w_post, w_pre, _ = data(3, 300, "f32", "f32")
    norm = BlockNorm(300, w_post, w_pre)
    cx, cn = norm.leave(xs, ys)
    ys[1, 5] = float("nan")
    gx, gn = norm.leave(xs, ys)
    assert torch.equal(gx[[0, 2]], cx[[0, 2]]) and torch.equal(gn[[0, 2]], cn[[0, 2]])
    assert torch.isnan(gx[1]).all() and torch.isnan(gn[1]).all()


def test_python_refusals():
    from paper_2608_21614_b200 import binding as B
    from paper_2608_21614_b200.norms import BlockNorm
    x, w = torch.zeros(4, 64, device="cuda"), torch.ones(64, device="cuda")
    norm, gated = BlockNorm(64, w, w), BlockNorm(64, w, w, gate="token")
    for call in (lambda: BlockNorm(64, w[:63]), lambda: BlockNorm(64, w, w.bfloat16()), lambda: norm.leave(x, x[:3]),
                 lambda: norm.leave(x, x, gate=x), lambda: gated.leave(x, x), lambda: gated.leave(x, x, gate=x),
                 lambda: norm.leave(x, x.half()), lambda: norm.leave(x.t(), x.t()), lambda: norm.leave(x, x, x_out=x.bfloat16())):
        with pytest.raises(B.SaemError):
            call()
