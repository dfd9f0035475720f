"""The 4-bit expert step for up to 8 tokens where its launches look different from the common case, against the 64-bit
reference of test_gpu_mx.py (same tolerances)."""
import numpy as np
import pytest
import torch

from test_gpu_mx import build, check_step

pytestmark = pytest.mark.gpu


def tokens(rng, T, d):
    return torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).cuda().to(torch.bfloat16)


@pytest.mark.parametrize("T", range(2, 9))
def test_far_fewer_active_experts_than_the_grid_allows_for(T):
    """Every token on the same eight experts, or on one that is there: most CTAs of the first launch have no item."""
    layer, exact, rng = build(1024, 256, 32, 8, T, seed=T)
    x = tokens(rng, T, 1024)
    logits = torch.full((T, 32), -2.0, device="cuda")
    logits[:, 3:27:3] = torch.from_numpy(rng.standard_normal((T, 8)).astype(np.float32)).cuda()
    first = check_step(layer, exact, logits, x, T)
    again = torch.empty_like(first)
    for _ in range(50):
        again.fill_(float("nan"))
        layer.step_fused_call(logits, x, T, again)
        assert torch.equal(first, again)
    layer.close()
