"""Tensors of the 4-bit operators and the norms that a kernel could not read -- on the host, of another type, too short -- are
refused before anything is launched.  (A launch on them would be a fault on the GPU.)"""
import pytest
import torch

from paper_2608_21614_b200 import binding as B
from paper_2608_21614_b200 import mx, norms

gpu = pytest.mark.gpu


def refused(call, code=B.SAEM_ERR_INVALID_ARG):
    with pytest.raises(B.SaemError) as e:
        call()
    assert e.value.code == code


def on_host(rows, cols):
    return mx.empty(rows, cols, device="cpu")


def test_weights_on_the_host_are_refused_when_the_operator_is_made():
    w = torch.ones(64)
    refused(lambda: norms.BlockNorm(64, w_pre=w))
    refused(lambda: norms.BlockNorm(64, w_post=w))
    refused(lambda: norms.BlockNorm(64, gate="row"))
    refused(lambda: mx.Linear(on_host(8, 64), 4))


@gpu
def test_quantised_matrices_on_the_host():
    x = torch.randn(4, 64, device="cuda")
    q, host, out = mx.quantize(x), on_host(4, 64), torch.full((4, 4), 7.0, device="cuda")
    refused(lambda: mx.quantize(x, out=host))
    refused(lambda: mx.dequantize(host, out=x))
    refused(lambda: mx.matmul(q, host, out=out))
    refused(lambda: mx.matmul(host, q, out=out))
    half = mx.MxTensor(4, 64, q.codes, host.scales)
    refused(lambda: mx.matmul(q, half, out=out))
    refused(lambda: mx.Linear(half, 4))
    linear = mx.Linear(q, 4)
    linear.weight = host
    refused(lambda: linear(x, out=out))
    linear.weight, linear.workspace = q, linear.workspace.cpu()
    refused(lambda: linear(x, out=out))
    torch.cuda.synchronize()
    assert (out == 7).all()


@gpu
def test_status_words_that_are_none():
    x = torch.randn(4, 64, device="cuda")
    q = mx.quantize(x)
    for status in (torch.zeros(1, dtype=torch.int32), torch.zeros(4, dtype=torch.uint8, device="cuda"), torch.zeros(1, device="cuda"),
                   torch.zeros(1, dtype=torch.int64, device="cuda")):
        refused(lambda: mx.matmul(q, q, status=status))
    refused(lambda: mx.matmul(q, q, status=torch.zeros(0, dtype=torch.int32, device="cuda")), B.SAEM_ERR_SHAPE)


@gpu
def test_weights_and_gates_of_a_norm():
    x, w = torch.randn(4, 64, device="cuda"), torch.ones(64, device="cuda")
    for bad, code in ((w.cpu(), B.SAEM_ERR_INVALID_ARG), (w.bfloat16(), B.SAEM_ERR_INVALID_ARG), (w[:63], B.SAEM_ERR_SHAPE),
                      (torch.ones(128, device="cuda")[::2], B.SAEM_ERR_INVALID_ARG)):
        norm = norms.BlockNorm(64, w_post=w, w_pre=w)
        norm.w_pre = bad
        refused(lambda: norm.enter(x), code)
        norm.w_pre, norm.w_post = w, bad
        refused(lambda: norm.leave(x, x), code)
    for kind, gate in (("token", torch.ones(4)), ("channel", torch.ones(64)), ("full", torch.ones(4, 64))):
        refused(lambda: norms.BlockNorm(64, w, w, gate=kind).leave(x, x, gate=gate))
    refused(lambda: norms.BlockNorm(64, w, w).leave(x, x.cpu()))


@gpu
def test_experts_and_routers_on_the_host():
    from paper_2608_21614_b200.layer import MoELayer
    from paper_2608_21614_b200.mx_block import MxMoEStack
    layer = MoELayer(128, 128, 2, 1, 4, ffn_path=B.SAEM_FFN_MX)
    there, host = mx.quantize(torch.randn(128, 128, device="cuda")), on_host(128, 128)
    refused(lambda: layer.load_expert_mx(0, 0, 0, there, host, there))
    assert B.saem_cache_query(layer.ctx.handle, 0, 0)[0] < 0
    layer.close()
    r = lambda *s: torch.randn(*s, device="cuda").bfloat16()                     # noqa: E731
    experts = [[(r(128, 128), r(128, 128), r(128, 128)) for _ in range(2)]]
    for router in (r(2, 128).cpu(), r(2, 128).float(), r(2, 127), r(128, 2).t()):
        refused(lambda: MxMoEStack(experts, [router], [r(128)], [r(128), r(128)], r(64, 128), 1, 4))


@gpu
def test_the_call_goes_to_the_stream_that_is_current():
    x = torch.randn(300, 512, device="cuda")
    want = mx.dequantize(mx.quantize(x))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = mx.dequantize(mx.quantize(x))
        side.synchronize()
    assert torch.equal(got, want)
