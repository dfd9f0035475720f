"""Calls of the 4-bit operators and the norms on a stream that is named and not the current one: what they allocate must not be
memory that earlier work of the current stream still uses."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def late_write(shape, dtype):
    """A buffer given back to the allocator while the current stream will still write to it, some milliseconds from now."""
    buf = torch.empty(shape, dtype=dtype, device="cuda")
    torch.cuda._sleep(40_000_000)
    buf.fill_(1)
    return buf.data_ptr()


def cases():
    from paper_2608_21614_b200 import mx, norms
    x = torch.randn(512, 2048, device="cuda")
    q = mx.quantize(x)
    linear = mx.Linear(q, 512)
    norm = norms.BlockNorm(2048)
    return {
        "dequantize": ((512, 2048), torch.float32, lambda st: mx.dequantize(q, stream=st)),
        "quantize": ((512 * 1024,), torch.uint8, lambda st: mx.quantize(x, stream=st).codes),
        "matmul": ((512, 512), torch.bfloat16, lambda st: mx.matmul(q, q, stream=st)),
        "linear": ((512, 512), torch.bfloat16, lambda st: linear(x, stream=st)),
        "enter": ((512, 2048), torch.bfloat16, lambda st: norm.enter(x, stream=st)),
        "leave": ((512, 2048), torch.float32, lambda st: norm.leave(x, x, stream=st)[0]),
    }


@pytest.mark.parametrize("named_by", ["stream", "handle"])
@pytest.mark.parametrize("name", ["dequantize", "quantize", "matmul", "linear", "enter", "leave"])
def test_results_of_a_named_stream_keep_clear_of_the_current_one(name, named_by):
    shape, dtype, call = cases()[name]
    want = call(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda.empty_cache()
    late_write(shape, dtype)
    got = call(side if named_by == "stream" else side.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_the_default_stream_by_its_handle():
    shape, dtype, call = cases()["dequantize"]
    assert torch.equal(call(0), call(None))


def test_the_status_word_waits_for_calls_on_every_stream():
    from paper_2608_21614_b200 import mx
    linear = mx.Linear(mx.quantize(torch.randn(64, 64, device="cuda")), 4)
    torch.zeros(1, dtype=torch.int32, device="cuda").fill_(3)           # loading the kernel would wait for the GPU
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):                                       # as a call would that runs out of time late
        torch.cuda._sleep(40_000_000)
        linear.workspace[:4].view(torch.int32).fill_(7)
    assert linear.device_status() == 7
