"""The 4-bit MoE stack (norm, router, expert step, norm, head) against the same chain in 64 bits, layer by layer.

A layer's reference starts from the GPU's own inputs of that layer.  Of the expert step, whose result y is fp32, the
hidden activations and x are held to 2^-13.8 of the largest of 32 neighbours: 2^-11 of |Wd| |h| bounds it (as in
test_gpu_mx.py), and the norms multiply y's error by no more than their own gain 1 / rms(y)."""
import numpy as np
import pytest
import torch

import mx_reference as ref

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def build(d, f, E, k, L, T, gated, seed=3):
    from paper_2608_21614_b200.mx_block import MxMoEStack
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device="cuda") * scale).to(torch.bfloat16)      # noqa: E731
    experts = [[(r(f, d, scale=d ** -0.5), r(f, d, scale=d ** -0.5), r(d, f, scale=f ** -0.5)) for _ in range(E)] for _ in range(L)]
    routers = [r(E, d, scale=d ** -0.5) for _ in range(L)]
    posts, pres = [1 + 0.1 * r(d) for _ in range(L)], [1 + 0.1 * r(d) for _ in range(L + 1)]
    gates = [r(d) for _ in range(L)] if gated else None
    head = r(384, d, scale=d ** -0.5)
    stack = MxMoEStack(experts, routers, posts, pres, head, k, T, branch_scale=0.5, gate=gates)
    return stack, experts, routers, posts, pres, gates, head


@pytest.mark.parametrize("T,gated", [(1, False), (6, True), (20, False)])
def test_stack_layer_by_layer(T, gated):
    d, f, E, k, L = 256, 384, 8, 2, 3
    stack, experts, routers, posts, pres, gates, head = build(d, f, E, k, L, T, gated)
    x = torch.randn(T, d, device="cuda") * 2
    stack.first.enter(x, n_out=stack.n[:T])
    assert np.abs(f64(stack.n[:T]) - ref.block_norm(f64(x), w_pre=f64(pres[0]))[1]).max() <= 2.0 ** -8 * 8
    for l in range(L):
        n, x0 = f64(stack.n[:T]), f64(x)
        stack.block(l, x)
        logits = f64(stack.logits[:T])
        assert np.abs(logits - n @ f64(routers[l]).T).max() <= 1e-4
        order = np.argsort(-logits, -1, kind="stable")[:, :k]
        top = np.take_along_axis(logits, order, -1)
        w = np.exp(top - top.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        mats = [[ref.quantize(f64(experts[l][e][i]))[0] for e in range(E)] for i in range(3)]
        y, bound = ref.moe(n, order, w, *mats)
        got_y = f64(stack.y[:T])
        assert (np.abs(got_y - y) <= 2.0 ** -11 * bound).all()
        want_x, want_n, size = ref.block_norm(x0, got_y, None if gates is None else f64(gates[l])[None], False, f64(posts[l]), f64(pres[l + 1]), b=0.5)
        assert (np.abs(f64(x) - want_x) <= 2.0 ** -20 * size).all()
        assert (np.abs(f64(stack.n[:T]) - want_n) <= 2.0 ** -8 * 1.01 * np.abs(want_n) + 1e-5).all()
    out = stack.head(stack.n[:T], out=stack.vocabulary[:T])
    a, b = ref.quantize(f64(stack.n[:T]))[0], ref.quantize(f64(head))[0]
    assert (np.abs(f64(out) - a @ b.T) <= 16 * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)).all()
    assert stack.device_status() == 0
    stack.close()


def test_stack_as_a_graph():
    stack, *_ = build(256, 256, 8, 2, 2, 4, False)
    x = torch.randn(4, 256, device="cuda")
    x0 = x.clone()
    graph = stack.capture(x)
    assert torch.equal(x, x0)
    graph.replay()
    torch.cuda.synchronize()
    got, got_x = stack.vocabulary[:4].clone(), x.clone()
    x.copy_(x0)
    want = stack.step(x)
    assert torch.equal(got, want) and torch.equal(got_x, x)
    stack.close()
