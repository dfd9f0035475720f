"""The inner-loop calls from Python without ctypes: what they refuse before anything reaches a GPU."""
import pytest
import torch

from paper_2608_21614_b200 import _host_calls as calls
from paper_2608_21614_b200 import binding as B
from paper_2608_21614_b200 import mx, norms


def test_wrong_numbers_and_kinds_of_arguments_are_type_errors():
    t = torch.zeros(2, 32)
    for f, n in ((calls.quantize, 6), (calls.dequantize, 6), (calls.matmul, 10), (calls.linear, 9), (calls.block_norm, 9)):
        with pytest.raises(TypeError):
            f(*[t] * (n - 1))
        with pytest.raises(TypeError):
            f(*[None] * n)
        with pytest.raises(TypeError):
            f(*["x"] * n)


def test_tensors_that_are_not_on_a_gpu_are_refused():
    q = mx.MxTensor(2, 32, torch.zeros(32, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8))
    x, y = torch.zeros(2, 32), torch.zeros(2, 32, dtype=torch.bfloat16)
    n = norms.BlockNorm(32)
    for f in (lambda: mx.quantize(x, out=q), lambda: mx.quantize(x), lambda: mx.dequantize(q, out=x), lambda: mx.matmul(q, q, out=y),
              lambda: n.enter(x, n_out=y), lambda: n.leave(x, y, x_out=x, n_out=y)):
        with pytest.raises(B.SaemError) as e:
            f()
        assert e.value.code == B.SAEM_ERR_INVALID_ARG


def test_a_configuration_of_another_size_is_refused():
    x = torch.zeros(2, 32)
    with pytest.raises(TypeError):
        calls.block_norm(b"\0" * 8, x, None, None, None, None, None, x, None)
