"""The attention half of a decoder layer and the stack with it: projections, head norms and rotation, cache, attention, norms.

Each step's reference starts from the GPU's own inputs of that step, with the bounds of the operators' own tests."""
import numpy as np
import pytest
import torch

import attention_reference as aref
import mx_reference as ref

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def weights(d, hq, hk, dim, seed=5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device="cuda") * scale).to(torch.bfloat16)      # noqa: E731
    return {"w_qkv": r((hq + 2 * hk) * dim, d, scale=d ** -0.5), "w_out": r(d, hq * dim, scale=(hq * dim) ** -0.5), "post": 1 + 0.1 * r(d), "pre": 1 + 0.1 * r(d),
            "w_q": 1 + 0.1 * r(dim), "w_k": 1 + 0.1 * r(dim)}


def layer(w, hq, hk, dim, pages, page, T, window=0, share=None):
    from paper_2608_21614_b200 import attention, rotary
    from paper_2608_21614_b200.mx_block import MxAttention
    cache = attention.PagedCache(*(torch.full((pages, hk, page, dim), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    return MxAttention(w["w_qkv"], w["w_out"], w["post"], w["pre"], cache, hq, T, rotary=rotary.Rotary(dim), w_q=w["w_q"], w_k=w["w_k"], window=window, share=share)


def batch_of(news, lengths, table):
    from paper_2608_21614_b200 import attention
    t = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")                                          # noqa: E731
    return attention.Batch(t([sum(news[:s]) for s in range(len(news) + 1)]), t(lengths), t(table), max_new=max(news))


@pytest.mark.parametrize("hq,hk,dim,page,window", [(8, 2, 64, 16, 0), (6, 2, 96, 32, 20), (4, 4, 128, 64, 0)])
def test_step_by_step(hq, hk, dim, page, window):
    from paper_2608_21614_b200 import rotary
    d, u = 256, 2.0 ** -8
    w = weights(d, hq, hk, dim)
    table = [[3, 0, 7], [5, 1, 2]]
    att = layer(w, hq, hk, dim, 8, page, 48, window)
    batch = batch_of([30, 11], [30, 11], table)
    x = torch.randn(41, d, device="cuda") * 2
    n = torch.randn(41, d, device="cuda").bfloat16()
    x0, n0 = f64(x), f64(n)
    att(x, n, batch)
    qkv = att.projected[:41]
    a, b = ref.quantize(n0)[0], ref.quantize(f64(w["w_qkv"]))[0]
    want, size = a @ b.T, np.abs(a) @ np.abs(b).T
    assert (np.abs(f64(qkv).reshape(41, -1) - want) <= u * np.abs(want) + 16 * 2.0 ** -23 * size).all()
    places = torch.cat((torch.arange(30), torch.arange(11))).cuda()
    f = rotary.frequencies(dim)[0]
    q = aref.rotation(qkv[:, :hq], places, f, w=w["w_q"])
    pairs = torch.sqrt(q[..., :dim // 2] ** 2 + q[..., dim // 2:] ** 2).repeat(1, 1, 2)
    assert bool(((att.rotated[:41].double() - q).abs() <= u * q.abs() + 2.0 ** -20.5 * pairs).all())
    t0 = 0
    for s, m in enumerate((30, 11)):
        pages = torch.tensor(table[s], device="cuda")
        k, v = (aref.gather(c, pages, m, page) for c in (att.attention.cache.k, att.attention.cache.v))
        assert torch.equal(v, qkv[t0:t0 + m, hq + hk:].transpose(0, 1))
        rk = aref.rotation(qkv[t0:t0 + m, hq:hq + hk], places[t0:t0 + m], f, w=w["w_k"]).transpose(0, 1)
        pairs = torch.sqrt(rk[..., :dim // 2] ** 2 + rk[..., dim // 2:] ** 2).repeat(1, 1, 2)
        assert bool(((k.double() - rk).abs() <= u * rk.abs() + 2.0 ** -20.5 * pairs).all())
        o, size, _, spread = aref.attend(att.rotated[t0:t0 + m], k, v, m, True, window, dim ** -0.5)
        delta = spread * ((dim + 8) * 2.0 ** -24 + 2.0 ** -22)
        assert bool(((att.weighted[t0:t0 + m].double() - o).abs() <= u * o.abs() + (u + 2 * delta[..., None] + 2.0 ** -18) * size).all())
        t0 += m
    a, b = ref.quantize(f64(att.weighted[:41]).reshape(41, -1))[0], ref.quantize(f64(w["w_out"]))[0]
    assert (np.abs(f64(att.y[:41]) - a @ b.T) <= 16 * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)).all()
    want_x, want_n, size = ref.block_norm(x0, f64(att.y[:41]), None, False, f64(w["post"]), f64(w["pre"]))
    assert (np.abs(f64(x) - want_x) <= 2.0 ** -20 * size).all()
    assert (np.abs(f64(n) - want_n) <= u * 1.01 * np.abs(want_n) + 1e-5).all()
    assert att.device_status() == 0


def test_a_prompt_at_once_in_chunks_and_token_by_token():
    """The attended tokens are the same within what the two orders of the sums and the weights' rounding leave: twice the bound of one."""
    hq, hk, dim, page, d, L = 8, 2, 64, 16, 256, 150
    w = weights(d, hq, hk, dim)
    table = [list(range(10))]
    ns = torch.randn(L, d, device="cuda").bfloat16()
    got, q, caches = [], [], []
    for steps in ([L], [64, 50, 36], [100] + [1] * 50):
        att = layer(w, hq, hk, dim, 10, page, L)
        at, parts, qs = 0, [], []
        for m in steps:
            x, n = torch.zeros(m, d, device="cuda"), ns[at:at + m].clone()
            at += m
            att(x, n, batch_of([m], [at], table))
            parts.append(att.weighted[:m].clone())
            qs.append(att.rotated[:m].clone())
        got.append(torch.cat(parts))
        q.append(torch.cat(qs))
        caches.append((att.attention.cache.k.clone(), att.attention.cache.v.clone()))
        assert att.device_status() == 0
    # the projections split their sums by the number of tokens: q, k and v may differ by a rounding, so each is compared with the formula over its own
    for o, rotated, (k, v) in zip(got, q, caches):
        k, v = (aref.gather(c, torch.arange(10, device="cuda"), L, page) for c in (k, v))
        want, size, _, spread = aref.attend(rotated, k, v, L, True, 0, dim ** -0.5)
        delta = spread * ((dim + 8) * 2.0 ** -24 + 2.0 ** -22)
        assert bool(((o.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2 * delta[..., None] + 2.0 ** -18) * size).all())
    for a in q[1:]:
        assert bool(((a.double() - q[0].double()).abs() <= 2.0 ** -4 * q[0].double().abs().amax(-1, keepdim=True)).all())


def stack(n_layers, T, pages, page, seed=1):
    from paper_2608_21614_b200.mx_block import random_stack
    return random_stack(256, 256, 8, 2, n_layers, 384, T, seed=seed, heads=(8, 2, 64), pages=pages, page_size=page)


def test_stack_with_attention_as_a_graph_while_lengths_grow():
    """Decode steps replayed from one graph, as the same steps called one by one."""
    xs = torch.randn(4, 3, 256, device="cuda")
    table = [[0, 1, 2], [3, 4, 5], [6, 7, 8]]
    results = []
    for captured in (False, True):
        s = stack(2, 3, 9, 16)
        for a in s.attention:
            g = torch.Generator(device="cuda").manual_seed(9)
            for c in (a.attention.cache.k, a.attention.cache.v):
                c.normal_(generator=g)
        batch = batch_of([1, 1, 1], [14, 1, 30], table)
        x, out = xs[0].clone(), []
        graph = s.capture(x, batch) if captured else None
        for i in range(4):
            x.copy_(xs[i])
            if captured:
                graph.replay()
            else:
                s.step(x, batch)
            out.append((s.vocabulary[:3].clone(), x.clone()))
            batch.lengths.add_(1)
        assert s.device_status() == 0
        results.append(out)
        s.close()
    for (a, b), (c, d) in zip(*results):
        assert torch.equal(a, c) and torch.equal(b, d)
    assert not torch.equal(results[0][0][0], results[0][1][0])


def test_layers_share_workspaces_and_refuse_other_shapes():
    from paper_2608_21614_b200 import attention, binding as B
    from paper_2608_21614_b200.mx_block import MxAttention, MxMoEStack
    s = stack(3, 4, 4, 16)
    a = s.attention
    assert a[0].attention.workspace.data_ptr() == a[2].attention.workspace.data_ptr() and a[0].rotated.data_ptr() == a[1].rotated.data_ptr()
    assert a[0].attention.cache.k.data_ptr() != a[1].attention.cache.k.data_ptr()
    x = torch.zeros(4, 256, device="cuda")
    with pytest.raises(B.SaemError):
        s.step(x)                                                               # a batch is wanted
    w = weights(256, 8, 2, 64)
    for bad in (dict(hq=4), dict(T=8)):
        kw = dict(hq=8, hk=2, dim=64, pages=4, page=16, T=4)
        kw.update(bad)
        with pytest.raises(B.SaemError):
            layer(w, share=a[0], **kw)
    half = attention.PagedCache.empty(2, 2, 16, 64, dtype=torch.float16)
    with pytest.raises(B.SaemError) as e:
        MxAttention(w["w_qkv"], w["w_out"], w["post"], w["pre"], half, 8, 4)
    assert e.value.code == B.SAEM_ERR_INVALID_ARG
    wide = attention.PagedCache.empty(2, 2, 16, 128)
    narrow = attention.Attention(8, attention.PagedCache.empty(2, 2, 16, 64))
    with pytest.raises(B.SaemError) as e:
        attention.Attention(8, wide, share=narrow)
    assert e.value.code == B.SAEM_ERR_WORKSPACE
    with pytest.raises(B.SaemError):
        MxMoEStack([[(w["pre"].expand(256, 256).contiguous(),) * 3] * 2], [torch.zeros(2, 256, device="cuda").bfloat16()], [w["post"]], [w["pre"]] * 2,
                   w["w_out"][:128, :256].contiguous(), 1, 4, attention=[])
    s.close()


def test_command_with_attention():
    import json
    import subprocess
    import sys
    out = subprocess.run([sys.executable, "-m", "paper_2608_21614_b200.mx_block", "--layers", "2", "--tokens", "2", "--steps", "3", "--d-model", "256", "--d-ff", "256",
                          "--experts", "8", "--top-k", "2", "--vocabulary", "512", "--context", "100", "--q-heads", "4", "--kv-heads", "2", "--head-dim", "64",
                          "--page-size", "16"], capture_output=True, text=True, timeout=240)
    assert out.returncode == 0, out.stderr[-2000:]
    line = json.loads(out.stdout.strip().splitlines()[-1])
    assert line["context"] == 100 and line["ms_per_step"] > 0
