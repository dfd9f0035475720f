"""The partially resident stack over 4-bit experts: misses through temporary slots against full residency and the 64-bit
reference (the tolerance of test_gpu_mx.py); host reads are refused when the runner is made."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from paper_2608_21614_b200 import binding as B
from paper_2608_21614_b200 import inputs as gen
from paper_2608_21614_b200.stack import StackRunner

L, E, K, D, F = 3, 8, 2, 256, 384


def test_host_reads_are_refused_when_the_runner_is_made():
    with pytest.raises(B.SaemError) as e:
        StackRunner(D, F, E, K, L, 4, 4, 4, [], ffn_path=B.SAEM_FFN_MX, miss_mode="host")
    assert e.value.code == B.SAEM_ERR_UNSUPPORTED


def run_stack(trace, weights, slots, temp, batch, steps):
    run = StackRunner(D, F, E, K, L, slots, temp, batch, weights, ffn_path=B.SAEM_FFN_MX)
    run.warm([list(np.argsort(trace.rankings[0, l])[:slots]) for l in range(L)])
    run.copy.synchronize()
    bounds, outs, inputs = set(int(b) for b in trace.boundaries[1:]), [], []
    for t in range(steps):
        if t in bounds:
            run.boundary()
        logits = np.stack([gen.trace_logits(trace, t, l, batch) for l in range(L)])
        x = gen.trace_activations(trace, t, batch, D)
        outs.append(run.step(torch.from_numpy(logits).cuda(), torch.from_numpy(x).cuda()).clone())
        inputs.append((logits, x))
    torch.cuda.synchronize()
    assert B.saem_last_device_status(run.h) == 0
    stats, store = run.stats, run.store
    run.close()
    return outs, inputs, stats, store


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 4, 12])
def test_half_of_the_experts_resident(batch):
    steps, rng = 24, np.random.default_rng(9)
    trace = gen.stage_trace(steps, L, E, 1.2, seed=5, mean_stage_len=8.0)
    weights = [gen.expert_weights(rng, D, F) for _ in range(6)]
    full, inputs, st_full, store = run_stack(trace, weights, E, 0, batch, steps)
    half, _, st_half, _ = run_stack(trace, weights, E // 2, 8, batch, steps)
    assert st_full.demand_loads == 0 and st_half.demand_loads > 0 and st_half.boundary_loads > 0
    for a, b in zip(full, half):
        assert torch.equal(a, b)                                        # placement changes no bit
    exact = [[ref.quantize(gen.bf16_bits_to_f32(w[i]))[0] for w in weights] for i in range(3)]
    for t in (0, steps - 1):
        logits, x = inputs[t]
        for l in range(L):
            order = np.argsort(-logits[l].astype(np.float64), -1, kind="stable")[:, :K]
            top = np.take_along_axis(logits[l].astype(np.float64), order, -1)
            w = np.exp(top - top.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            mats = [[m[store.index(l, e)] for e in range(E)] for m in exact]
            want, bound = ref.moe(gen.bf16_bits_to_f32(x).astype(np.float64), order, w, *mats)
            assert (np.abs(half[t][l].cpu().numpy() - want) <= 2.0 ** -11 * bound + 2.0 ** -140).all()
