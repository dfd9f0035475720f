"""Rows of a layer's and a stack's call that belong to no sequence."""
import math

import pytest
import torch

import test_gpu_mx_attention as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [2, 45])
@pytest.mark.parametrize("spare", ["zero", "random", "nan"])
def test_spare_rows_do_not_reach_the_others(tokens, spare):
    """A step of more rows than its sequences have: the others' results and the caches are the same bits whatever the spare rows hold."""
    table = [[3, 0, 7, 9], [5, 1, 2, 4]]
    rows, results = tokens + 5, []
    for fill in ("ones", spare):
        s = base.stack(2, rows, 10, 16)
        for a in s.attention:
            g = torch.Generator(device="cuda").manual_seed(9)
            for c in (a.attention.cache.k, a.attention.cache.v):
                c.normal_(generator=g)
            for buffer in (a.projected, a.rotated, a.weighted):
                assert bool((buffer == 0).all())                                # nothing of what the memory held before
        g = torch.Generator(device="cuda").manual_seed(4)
        x = torch.randn(rows, 256, generator=g, device="cuda")
        x[tokens:] = {"ones": 1.0, "zero": 0.0, "nan": math.nan}.get(fill, 0.0)
        if fill == "random":
            x[tokens:] = 100 * torch.randn(5, 256, generator=g, device="cuda")
        n = tokens // 2
        for step in range(2):                                                   # the second with what the first left in the buffers
            out = s.step(x, base.batch_of([n, tokens - n], [n + 3 + step, tokens - n + 5 + step], table))
            x[tokens:].nan_to_num_(0.0) if fill != "nan" else x[tokens:].fill_(math.nan)
        results.append((out[:tokens].clone(), x[:tokens].clone(), *(c[[3, 0, 7, 9, 5, 1, 2, 4]].clone() for a in s.attention for c in (a.attention.cache.k, a.attention.cache.v))))
        assert s.device_status() == 0
        s.close()
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert bool(torch.isfinite(results[0][0]).all())
