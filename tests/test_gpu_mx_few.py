"""The 4-bit expert step for up to 8 tokens where its launches look different from the common case, against the 64-bit
reference of test_gpu_mx.py (same tolerances)."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from paper_2608_21614_b200 import inputs as gen
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


def build_of(d, f, E, k, T, distinct, seed=0, **kw):
    """As build(), with `distinct` different experts that take turns (large layers in little time)."""
    from paper_2608_21614_b200 import binding as B, mx
    from paper_2608_21614_b200.layer import MoELayer
    rng = np.random.default_rng(seed)
    layer = MoELayer(d, f, E, k, T, ffn_path=B.SAEM_FFN_MX, **kw)
    wide = [[torch.from_numpy(gen.bf16_bits_to_f32(m)) for m in gen.expert_weights(rng, d, f)] for _ in range(distinct)]
    exact = [[ref.quantize(m[i].numpy())[0] for m in wide] for i in range(3)]
    q = [[mx.quantize(m.cuda()) for m in ms] for ms in wide]
    for e in range(E):
        layer.load_expert_mx(0, e, e, *q[e % distinct])
    torch.cuda.synchronize()
    return layer, [[exact[i][e % distinct] for e in range(E)] for i in range(3)], rng


# d_model, d_ff, experts, top_k, tokens, different experts
FORMS = [
    (512, 1280, 32, 8, 8, 5),       # whole blocks, two or three items per CTA; 20 units of each down part, four stages
    (256, 768, 16, 8, 8, 5),        # halves, some CTAs with two items
    (640, 1152, 20, 8, 7, 4),       # whole blocks, odd numbers of 128 in both axes
    (4096, 128, 4, 2, 8, 4),        # sixteen runs of x, halves
    (3968, 128, 5, 3, 3, 5),        # the last run is half full
    (4096, 384, 64, 8, 8, 3),       # sixteen runs, whole blocks, a ring of three stages that goes round
    (3968, 384, 64, 8, 6, 3),
    (4096, 256, 8, 8, 1, 4),        # one token
    (256, 4096, 8, 4, 8, 4),        # long down projection
]


@pytest.mark.parametrize("d,f,E,k,T,distinct", FORMS)
def test_forms_of_the_two_launches(d, f, E, k, T, distinct):
    layer, exact, rng = build_of(d, f, E, k, T, distinct, seed=d + f)
    x = tokens(rng, T, d)
    x[:, 5] *= 30
    logits = torch.from_numpy(rng.standard_normal((T, E)).astype(np.float32)).cuda()
    for t in range(T):                                                  # as many experts as the tokens can reach
        logits[t, [(t * k + j) % E for j in range(k)]] += 6.0
    first = check_step(layer, exact, logits, x, T)
    again = torch.empty_like(first)
    for _ in range(5):
        again.fill_(float("nan"))
        layer.step_fused_call(logits, x, T, again)
        assert torch.equal(first, again)
    layer.close()


@pytest.mark.parametrize("d,f,E,k,T", [(4224, 128, 4, 2, 1), (4224, 256, 4, 2, 8), (8192, 128, 3, 2, 3), (256, 256, 16, 12, 5), (256, 128, 16, 9, 8),
                                       (256, 128, 20, 20, 1)])
def test_few_tokens_outside_the_two_launches(d, f, E, k, T):
    layer, exact, rng = build_of(d, f, E, k, T, 3, seed=d + k)
    logits = torch.from_numpy(rng.standard_normal((T, E)).astype(np.float32)).cuda()
    check_step(layer, exact, logits, tokens(rng, T, d), T)
    layer.close()


@pytest.mark.parametrize("T", [1, 8, 9, 40])
def test_a_shared_expert_of_another_width_in_a_second_context(T):
    from paper_2608_21614_b200 import binding as B
    from paper_2608_21614_b200.layer import MoELayer
    d, f, fs, E, k = 256, 256, 384, 4, 2
    rng = np.random.default_rng(T)
    layer = MoELayer(d, f, E, k, T, d_ff_shared=fs, ffn_path=B.SAEM_FFN_MX)
    assert layer.shared is not None
    mats = [gen.expert_weights(rng, d, f) for _ in range(E)] + [gen.expert_weights(rng, d, fs)]
    layer.load_all(*([m[i] for m in mats[:E]] for i in range(3)), shared=mats[E])
    layer.copy_stream.synchronize()
    exact = [[ref.quantize(gen.bf16_bits_to_f32(m[i]))[0] for m in mats] for i in range(3)]
    logits = torch.from_numpy(rng.standard_normal((T, E)).astype(np.float32)).cuda()
    x = tokens(rng, T, d)
    check_step(layer, exact, logits, x, T, S=1)
    whole = torch.empty(T, d, device="cuda")
    layer.step_fused_call(logits, x, T, whole)
    assert torch.equal(layer.step(logits, x, T), whole)                 # call by call: the same kernels
    layer.close()


@pytest.mark.parametrize("T", [4, 12])
@pytest.mark.parametrize("which", [0, 1, 2])
def test_an_expert_that_is_not_finite_reaches_its_own_tokens_only(which, T):
    """NaN in one row of one expert's gate, up or down matrix: the tokens of the other experts stay as they are."""
    from paper_2608_21614_b200 import binding as B, mx
    d, f, E = 256, 384, 4
    layer, exact, rng = build_of(d, f, E, 1, T, E, seed=3)
    x = tokens(rng, T, d)
    logits = torch.zeros(T, E, device="cuda")
    logits[torch.arange(T), torch.arange(T) % E] = 5.0                  # token t on expert t % 4
    clean = check_step(layer, exact, logits, x, T)
    mats = [torch.from_numpy(exact[i][2].astype(np.float32)).cuda() for i in range(3)]
    mats[which][7, 100] = float("nan")
    B.saem_cache_evict(layer.ctx.handle, 0, 2)
    layer.load_expert_mx(0, 2, 2, *(mx.quantize(m) for m in mats))
    torch.cuda.synchronize()
    out = torch.empty_like(clean)
    layer.step_fused_call(logits, x, T, out)
    own = torch.arange(T, device="cuda") % E == 2
    limit = 2.0 ** -18 * clean[~own].abs().max()                        # the same terms, another order of fp32 sums at most
    assert ((out[~own] - clean[~own]).abs() <= limit).all()
    bad = torch.isnan(out[own])
    want = torch.zeros_like(bad)
    if which == 2:
        want[:, 7] = True                                               # one output column
    else:
        want[:] = True                                                  # one hidden unit, hence every output
    assert torch.equal(bad, want)
    again = torch.empty_like(out)
    layer.step_fused_call(logits, x, T, again)
    assert torch.equal(out.view(torch.int32), again.view(torch.int32))
    layer.close()
