"""Head norms with rotation, and appending to a paged cache, against the formula in 64 bits.

Bounds: the angle's sine and cosine are off by 2^-22 (the argument in half turns to 2^-25, times pi; sincospi to a few 2^-24), the norm's
factor, the weights and the two products add at most 16 roundings of 2^-24, all relative to the size of the pair; then the result is rounded once (u = eps / 2)."""
import pytest
import torch

import attention_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def close(got, want, rotary_dim, interleaved, amplitude=1.0):
    """want float64; the size of a pair bounds both of its elements."""
    u = torch.finfo(got.dtype).eps / 2
    size = want.abs().clone()
    n = rotary_dim // 2
    if n:
        a, b = (want[..., 0:2 * n:2], want[..., 1:2 * n:2]) if interleaved else (want[..., :n], want[..., n:2 * n])
        r = torch.sqrt(a * a + b * b)
        if interleaved:
            size[..., 0:2 * n:2], size[..., 1:2 * n:2] = r, r
        else:
            size[..., :n], size[..., n:2 * n] = r, r
    off = (got.double() - want).abs() - (u * want.abs() + (2.0 ** -20.5) * size + torch.finfo(got.dtype).tiny)
    assert float(off.max()) <= 0, float(off.max())


@pytest.mark.parametrize("tokens,heads", [(1, 1), (1, 40), (3, 5), (77, 9), (2000, 3)])
@pytest.mark.parametrize("dim,rot", [(128, 128), (128, 64), (64, 64), (96, 48), (80, 80), (8, 8), (72, 8), (120, 0), (112, 104)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_sizes(tokens, heads, dim, rot, interleaved):
    from paper_2608_21614_b200 import rotary
    r = rotary.Rotary(dim, rot, interleaved=interleaved)
    x = torch.randn(tokens, heads, dim, generator=gen(tokens + dim), device="cuda").bfloat16()
    p = torch.randint(0, 4096, (tokens,), generator=gen(1), device="cuda", dtype=torch.int32)
    w = (1 + 0.2 * torch.randn(dim, generator=gen(2), device="cuda"))
    f, _ = rotary.frequencies(rot)
    close(r.rotate(x, p), ref.rotation(x, p, f, interleaved), rot, interleaved)
    close(r.rotate(x, p, weight=w, eps=1e-3), ref.rotation(x, p, f, interleaved, w=w, eps=1e-3), rot, interleaved)


@pytest.mark.parametrize("x_type", TYPES)
@pytest.mark.parametrize("out_type", TYPES)
@pytest.mark.parametrize("w_type", [torch.float32, torch.bfloat16])
def test_types(x_type, out_type, w_type):
    from paper_2608_21614_b200 import rotary
    r = rotary.Rotary(128, 96)
    x = torch.randn(19, 6, 128, generator=gen(0), device="cuda").to(x_type)
    p = torch.arange(100, 119, device="cuda", dtype=torch.int32)
    w = (1 + 0.2 * torch.randn(128, generator=gen(2), device="cuda")).to(w_type)
    got = r.rotate(x, p, weight=w, dtype=out_type)
    assert got.dtype == out_type
    close(got, ref.rotation(x, p, rotary.frequencies(96)[0], w=w), 96, False)


@pytest.mark.parametrize("scaling", [None, {"kind": "linear", "factor": 4.0}, {"kind": "base", "factor": 8.0},
                                     {"kind": "bands", "factor": 8.0, "original": 8192.0, "low": 1.0, "high": 4.0},
                                     {"kind": "yarn", "factor": 32.0, "original": 4096.0}])
def test_far_positions_and_scalings(scaling):
    """Positions up to 2^31: the angle is as exact there as near zero."""
    from paper_2608_21614_b200 import rotary
    r = rotary.Rotary(64, base=500000.0, scaling=scaling)
    f, amplitude = rotary.frequencies(64, 500000.0, scaling)
    p = torch.tensor([0, 1, 4095, 131071, 1 << 20, (1 << 24) + 1, 2 ** 31 - 1, -1, -(1 << 20)], dtype=torch.int32, device="cuda")
    x = torch.randn(len(p), 2, 64, generator=gen(0), device="cuda")
    # p f in float64 is off by p f 2^-53: 2^-22 of a radian at 2^31
    close(r.rotate(x, p), ref.rotation(x, p, f, amplitude=amplitude), 64, False)


@pytest.mark.parametrize("offset", [0, 1, 2, 3, 4])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_alignment(offset, interleaved, dtype):
    """Heads that begin at any element, tokens and heads in either order, expanded heads; the result in place."""
    from paper_2608_21614_b200 import rotary
    r = rotary.Rotary(96, 48, interleaved=interleaved)
    f = rotary.frequencies(48)[0]
    p = torch.arange(7, 20, device="cuda", dtype=torch.int32)
    flat = torch.randn(13 * 5 * 101 + 8, generator=gen(3), device="cuda").to(dtype)
    for view in (flat[offset:offset + 13 * 5 * 101].view(13, 5, 101)[..., :96], flat[offset:offset + 13 * 5 * 101].view(5, 13, 101).transpose(0, 1)[..., :96],
                 flat[offset:offset + 13 * 101].view(13, 1, 101)[..., :96].expand(13, 5, 96)):
        want = ref.rotation(view, p, f, interleaved)
        close(r.rotate(view, p), want, 48, interleaved)
        keep = flat.clone()
        if view.stride(1):
            r.rotate(view, p, out=view)
            close(view, want, 48, interleaved)
            view.copy_(torch.as_strided(keep, view.shape, view.stride(), offset))
            assert torch.equal(flat, keep)              # and nothing beside it


def test_norm_of_odd_values():
    """Zeros, huge and tiny rows, an infinity and a NaN stay in their head."""
    from paper_2608_21614_b200 import rotary
    r = rotary.Rotary(64)
    x = torch.ones(6, 2, 64, device="cuda")
    x[0, 0] = 0
    x[1, 0] = 1e18
    x[2, 0] = 1e-30
    x[3, 0, 3] = float("inf")
    x[4, 0, 3] = float("nan")
    p = torch.arange(6, device="cuda", dtype=torch.int32)
    w = torch.ones(64, device="cuda")
    got = r.rotate(x, p, weight=w)
    want = ref.rotation(x, p, rotary.frequencies(64)[0], w=w)
    rows = [0, 1, 2, 5]
    close(got[rows], want[rows], 64, False)
    close(got[:, 1], want[:, 1], 64, False)
    assert bool(torch.isnan(got[3, 0]).any()) and bool(torch.isnan(got[4, 0]).all())


def batch_of(seqs, page, pages, seed=0, extra=1):
    from paper_2608_21614_b200 import attention
    need = [-(-n // page) for _, n in seqs]
    order = torch.randperm(pages, generator=gen(seed), device="cuda").int()
    table = torch.full((len(seqs), max(need + [1]) + extra), 1 << 30, dtype=torch.int32, device="cuda")
    at, offsets = 0, [0]
    for s, (m, _) in enumerate(seqs):
        table[s, :need[s]] = order[at:at + need[s]]
        at += need[s]
        offsets.append(offsets[-1] + m)
    assert at <= pages
    return attention.Batch(torch.tensor(offsets, dtype=torch.int32, device="cuda"), torch.tensor([n for _, n in seqs], dtype=torch.int32, device="cuda"),
                           table, max_new=max(m for m, _ in seqs)), offsets


SEQS = {"one": [(1, 1)], "decode": [(1, 17 + 13 * s) for s in range(19)], "chunk": [(333, 900)], "ragged": [(5, 5), (0, 40), (64, 200), (1, 63), (0, 0), (17, 18)],
        "many": [(s % 3, 3 + s % 50) for s in range(1200)], "fewer places than tokens": [(9, 4), (2, 0), (3, 3)]}


@pytest.mark.parametrize("shape", list(SEQS))
@pytest.mark.parametrize("x_type,cache_type", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16), (torch.float32, torch.float16), (torch.float16, torch.bfloat16)])
@pytest.mark.parametrize("dim,rot,page,interleaved,normed", [(128, 128, 64, False, True), (96, 48, 16, True, False), (64, 0, 48, False, True), (72, 72, 32, False, True)])
def test_append(shape, x_type, cache_type, dim, rot, page, interleaved, normed):
    from paper_2608_21614_b200 import attention, rotary
    seqs, hq, hk = SEQS[shape], 6, 2
    pages = sum(-(-n // page) for _, n in seqs) + 4
    batch, offsets = batch_of(seqs, page, pages)
    T = offsets[-1] + 3                                                         # three rows behind the last sequence
    g = gen(7)
    cache = attention.PagedCache(*(torch.randn(pages, hk, page, dim, generator=g, device="cuda").to(cache_type) for _ in range(2)))
    want_k, want_v = cache.k.double(), cache.v.double()
    keep_k, keep_v = cache.k.clone(), cache.v.clone()
    qkv = torch.randn(T, hq + 2 * hk, dim, generator=g, device="cuda").to(x_type)
    q, k, v = qkv.split([hq, hk, hk], 1)
    w_q, w_k = (((1 + 0.1 * torch.randn(dim, generator=g, device="cuda")).bfloat16() if normed else None) for _ in range(2))
    turn = rotary.Rotary(dim, rot, interleaved=interleaved)
    f = rotary.frequencies(rot)[0]
    att = attention.Attention(hq, cache, rotary=turn, w_q=w_q, w_k=w_k, eps=1e-5)
    q_out = torch.full((T, hq, dim), 5.0, dtype=cache_type, device="cuda")
    att.append(q, k, v, batch, q_out=q_out)
    assert att.device_status() == 0
    places = torch.cat([torch.arange(n - m, n) for m, n in seqs]).cuda()
    seq = torch.cat([torch.full((m,), s) for s, (m, _) in enumerate(seqs)]).cuda()
    n = len(places)
    close(q_out[:n], ref.rotation(q[:n], places, f, interleaved, w=w_q, eps=1e-5), rot, interleaved)
    assert bool((q_out[n:] == 5).all())
    rk = ref.rotation(k[:n], places, f, interleaved, w=w_k, eps=1e-5)
    stored = places >= 0
    page_of, slot = batch.table[seq[stored], (places[stored] // page)].long(), places[stored] % page
    close(cache.k[page_of, :, slot], rk[stored], rot, interleaved)
    assert torch.equal(cache.v[page_of, :, slot], v[:n][stored].float().to(cache_type))
    keep_k[page_of, :, slot], keep_v[page_of, :, slot] = cache.k[page_of, :, slot], cache.v[page_of, :, slot]
    assert torch.equal(cache.k, keep_k) and torch.equal(cache.v, keep_v)        # no other place


def test_append_with_positions_without_rotation_without_queries():
    from paper_2608_21614_b200 import attention, rotary
    batch, _ = batch_of([(4, 40), (2, 10)], 16, 8)
    g = gen(1)
    k, v = (torch.randn(6, 2, 64, generator=g, device="cuda").bfloat16() for _ in range(2))
    cache = attention.PagedCache.empty(8, 2, 16, 64)
    att = attention.Attention(4, cache, rotary=rotary.Rotary(64))
    p = torch.tensor([9, 1, 70000, 3, 0, 5], dtype=torch.int32, device="cuda")
    assert att.append(None, k, v, batch, positions=p) is None
    places, seq = torch.tensor([36, 37, 38, 39, 8, 9]).cuda(), torch.tensor([0, 0, 0, 0, 1, 1]).cuda()
    at = batch.table[seq, places // 16].long(), places % 16
    close(cache.k[at[0], :, at[1]], ref.rotation(k, p, rotary.frequencies(64)[0]), 64, False)
    plain = attention.Attention(2, cache)                                       # neither norm nor rotation
    q = torch.randn(6, 2, 64, generator=g, device="cuda").bfloat16()
    assert torch.equal(plain.append(q, k, v, batch), q)
    assert torch.equal(cache.k[at[0], :, at[1]], k) and torch.equal(cache.v[at[0], :, at[1]], v)


def test_places_without_a_page_are_not_stored():
    from paper_2608_21614_b200 import attention, binding as B
    for bad in (-1, 5, 2 ** 31 - 1, None):
        batch, _ = batch_of([(3, 20), (2, 33)], 16, 5, extra=0)
        cache = attention.PagedCache(*(torch.zeros(5, 2, 16, 64, device="cuda").bfloat16() for _ in range(2)))
        if bad is None:
            batch.lengths[1] = 49                                               # its last place is behind the table
        else:
            batch.table[1, 2] = bad
        att = attention.Attention(2, cache)
        x = torch.ones(5, 2, 64, device="cuda").bfloat16()
        att.append(None, x, x, batch)
        assert att.device_status() == B.SAEM_ERR_INVALID_ARG
        assert int((cache.k[:, 0, :, 0] != 0).sum()) == 4                       # all tokens but one


def test_captured_append_and_attend_on_a_named_stream():
    """One decode step, appended and attended, captured once and replayed for further tokens: as step by step."""
    from paper_2608_21614_b200 import attention, rotary
    g = gen(11)
    steps, S, hq, hk, dim = 5, 3, 4, 2, 64
    x = torch.randn(steps, S, hq + 2 * hk, dim, generator=g, device="cuda").bfloat16()

    def fresh():
        batch, _ = batch_of([(1, 30), (1, 1), (1, 15)], 16, 12, extra=2)
        batch.table[batch.table > 12] = 11
        batch.table[1, 1], batch.table[2, 1] = 9, 10
        cache = attention.PagedCache(*(torch.randn(12, hk, 16, dim, generator=gen(12), device="cuda").bfloat16() for _ in range(2)))
        return batch, cache, attention.Attention(hq, cache, rotary=rotary.Rotary(dim))
    batch, cache, att = fresh()
    want = []
    for i in range(steps):
        q, k, v = x[i].split([hq, hk, hk], 1)
        want.append(att.attend(att.append(q, k, v, batch), batch).clone())
        batch.lengths += 1
    batch, cache, att = fresh()
    now, q_out, out = torch.empty_like(x[0]), torch.empty(S, hq, dim, dtype=torch.bfloat16, device="cuda"), torch.empty(S, hq, dim, dtype=torch.bfloat16, device="cuda")
    now.copy_(x[0])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    q, k, v = now.split([hq, hk, hk], 1)
    att.append(q, k, v, batch, q_out=q_out, stream=side)
    att.attend(q_out, batch, out=out, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        att.append(q, k, v, batch, q_out=q_out)
        att.attend(q_out, batch, out=out)
    for i in range(steps):
        now.copy_(x[i])
        graph.replay()
        assert torch.equal(out, want[i])
        batch.lengths += 1


def test_append_in_place():
    """q_out may be q itself; the cache gets what it gets otherwise."""
    from paper_2608_21614_b200 import attention, rotary
    g = gen(3)
    for interleaved in (False, True):
        batch, _ = batch_of([(9, 40), (1, 16), (30, 30)], 16, 9)
        qkv = torch.randn(40, 20, 80, generator=g, device="cuda").bfloat16()
        w = (1 + 0.1 * torch.randn(80, generator=g, device="cuda")).bfloat16()
        results = []
        for in_place in (False, True):
            cache = attention.PagedCache(*(torch.zeros(9, 2, 16, 80, device="cuda").bfloat16() for _ in range(2)))
            att = attention.Attention(16, cache, rotary=rotary.Rotary(80, 64, interleaved=interleaved), w_q=w, w_k=w)
            x = qkv.clone()
            q, k, v = x.split([16, 2, 2], 1)
            out = att.append(q, k, v, batch, q_out=q if in_place else None)
            results.append((out.clone(), cache.k, cache.v))
            assert torch.equal(x[:, 16:], qkv[:, 16:])
        assert all(torch.equal(a, b) for a, b in zip(*results))
