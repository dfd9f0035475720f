"""Attention over a paged cache, against the formula in 64 bits.

Bounds, with u = eps / 2 of the 16-bit type: the weights p are rounded to it before the second product (u * sum p |v|), the result
once more (u |out|); a score in fp32 is off by at most (dim + 8) 2^-24 of scale * sum |q| |k| and by 2^-22 of itself on the way into the
exponent, which changes a weight, and the sum of weights, by twice that; 2^-18 covers the exponentials and the sums over places.  A float16 weight
below 2^-24 is lost: 2^-25 of the largest value for each place."""
import math

import pytest
import torch

import attention_reference as ref

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def build(seqs, q_heads, kv_heads, dim, page, dtype, seed=0, garbage=float("nan"), spare_pages=3, spare_rows=None, table_extra=2):
    """seqs: (new, length) each.  A cache whose every place outside the sequences is `garbage`, and rows behind the last sequence: so many, unless
    said otherwise, that a call is none of few rows in all, and max_new alone chooses the form (1: few rows per key head, 1000: many)."""
    from paper_2608_21614_b200 import attention
    g = gen(seed)
    need = [-(-n // page) for _, n in seqs]
    pages = sum(need) + spare_pages
    order = torch.randperm(pages, generator=g, device="cuda").int()
    table = torch.full((len(seqs), max(need + [1]) + table_extra), -7, dtype=torch.int32, device="cuda")
    k, v = (torch.full((pages, kv_heads, page, dim), garbage, dtype=dtype, device="cuda") for _ in range(2))
    at = 0
    for s, (_, n) in enumerate(seqs):
        table[s, :need[s]] = order[at:at + need[s]]
        for c in (k, v):
            x = torch.full((kv_heads, need[s] * page, dim), garbage, device="cuda")
            x[:, :n] = torch.randn(kv_heads, n, dim, generator=g, device="cuda")
            c[order[at:at + need[s]].long()] = x.view(kv_heads, need[s], page, dim).transpose(0, 1).to(dtype)
        at += need[s]
    offsets = [0]
    for m, _ in seqs:
        offsets.append(offsets[-1] + m)
    rows = offsets[-1] + (800 // q_heads + 1 if spare_rows is None else spare_rows)
    q = (torch.randn(rows, q_heads, dim, generator=g, device="cuda") * 1.5).to(dtype)
    batch = attention.Batch(torch.tensor(offsets, dtype=torch.int32, device="cuda"), torch.tensor([n for _, n in seqs], dtype=torch.int32, device="cuda"),
                            table, max_new=max([m for m, _ in seqs] + [0]))
    return q, attention.PagedCache(k, v), batch, offsets


def check(out, lse, q, cache, batch, seqs, offsets, causal, window, scale):
    u = torch.finfo(q.dtype).eps / 2
    tiny = 2.0 ** -25 if q.dtype == torch.float16 else 0.0
    page, dim = cache.page_size, q.shape[2]
    for s, (n, length) in enumerate(seqs):
        if n == 0:
            continue
        t = slice(offsets[s], offsets[s + 1])
        k, v = (ref.gather(c, batch.table[s], length, page) for c in (cache.k, cache.v))
        want, size, want_lse, spread = ref.attend(q[t], k, v, n, causal, window, scale)
        got = out[t].double()
        delta = spread * ((dim + 8) * 2.0 ** -24 + 2.0 ** -22)
        finite = torch.nan_to_num(v.double(), 0.0, 0.0, 0.0)
        top = finite.abs().amax() if length else torch.zeros((), dtype=torch.float64, device="cuda")
        bound = u * want.abs() + (u + 2 * delta[..., None] + 2.0 ** -18) * size + tiny * length * top + torch.finfo(q.dtype).tiny * 2
        same = torch.isnan(want) == torch.isnan(got)
        assert bool(same.all()), "sequence %d: NaN in %d places, wanted in %d" % (s, int(torch.isnan(got).sum()), int(torch.isnan(want).sum()))
        good = torch.isfinite(want)
        off = ((got - want).abs() - bound)[good]
        assert off.numel() == 0 or float(off.max()) <= 0, (s, float(off.max()))
        assert torch.equal(got[~good & ~torch.isnan(want)], want[~good & ~torch.isnan(want)])
        if lse is not None:
            far = (lse[t].double() - want_lse).abs()
            seen = torch.isfinite(want_lse)
            assert bool((far[seen] <= (2 * delta + 2.0 ** -18 + 2.0 ** -22 * want_lse.abs())[seen]).all())
            assert torch.equal(lse[t].double()[~seen & ~torch.isnan(want_lse)], want_lse[~seen & ~torch.isnan(want_lse)])


def run(seqs, q_heads=8, kv_heads=2, dim=128, page=64, dtype=torch.bfloat16, causal=True, window=0, scale=None, max_new=None, seed=0, lse=True, **kw):
    from paper_2608_21614_b200 import attention
    q, cache, batch, offsets = build(seqs, q_heads, kv_heads, dim, page, dtype, seed, **kw)
    if max_new is not None:
        batch.max_new = max_new
    att = attention.Attention(q_heads, cache, causal=causal, window=window, scale=scale)
    out = torch.full_like(q, 77.0)
    l = torch.full((q.shape[0], q_heads), 55.0, device="cuda") if lse else None
    att.attend(q, batch, out=out, lse=l)
    assert att.device_status() == 0
    check(out, l, q, cache, batch, seqs, offsets, causal, window, dim ** -0.5 if scale is None else scale)
    assert bool((out[offsets[-1]:] == 77.0).all()) and (l is None or bool((l[offsets[-1]:] == 55.0).all()))
    assert bool((att.workspace[256:8192] == 0).all())
    return out


def test_few_rows_in_all():
    """As a program calls it, without rows to spare: up to 768 rows go to the form for few, one more to the other."""
    for new in (47, 48, 49):
        run([(new, 200), (48, 100)], q_heads=8, kv_heads=2, spare_rows=0)
    run([(300, 700)], q_heads=2, kv_heads=1, spare_rows=0)


# one new token, or a few
@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 500, 1000, 4097])
def test_one_token(length):
    run([(1, length)], q_heads=8, kv_heads=2)


@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (4, 4), (5, 1), (16, 1), (17, 1), (12, 4), (32, 4), (48, 2), (128, 1)])
@pytest.mark.parametrize("max_new", [1, 1000])
def test_heads(q_heads, kv_heads, max_new):
    run([(1, 333), (2, 70), (1, 1)], q_heads=q_heads, kv_heads=kv_heads, max_new=max_new)


@pytest.mark.parametrize("dim", [8, 16, 24, 64, 72, 80, 96, 104, 112, 120, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("max_new", [1, 1000])
def test_head_sizes(dim, dtype, max_new):
    run([(3, 301), (1, 64), (40, 200)], dim=dim, dtype=dtype, max_new=max_new)


@pytest.mark.parametrize("page", [16, 32, 48, 64, 80, 128, 144, 256, 4096])
@pytest.mark.parametrize("max_new", [1, 1000])
def test_pages(page, max_new):
    run([(1, 777), (9, 130), (200, 555)], page=page, max_new=max_new)


# long chunks, ragged, without tokens, without places
SHAPES = {
    "chunk": [(129, 129)],
    "chunk over a cache": [(257, 1500)],
    "whole tiles": [(256, 512)],
    "ragged": [(1, 900), (300, 300), (0, 50), (17, 18), (64, 1000), (0, 0), (1, 1), (600, 601)],
    "short": [(n, n) for n in range(1, 40)],
    "fewer places than tokens": [(20, 5), (3, 0), (200, 130), (1, 0), (5, 5)],
    "many": [(1 + s % 3, 1 + s * 7 % 97) for s in range(700)],
}


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("max_new", [1, 1000])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 100), (False, 33), (True, 1)])
def test_shapes_and_masks(shape, max_new, causal, window):
    run(SHAPES[shape], causal=causal, window=window, max_new=max_new)


@pytest.mark.parametrize("max_new", [1, 1000])
@pytest.mark.parametrize("seqs", [[(2, 40000)], [(130, 20000)], [(1, 30000), (1, 10), (40, 9000)]])
def test_long(seqs, max_new):
    run(seqs, q_heads=4, kv_heads=2, max_new=max_new)


@pytest.mark.parametrize("max_new", [1, 1000])
@pytest.mark.parametrize("scale", [1e-6, 0.3, 40.0])
def test_scales(scale, max_new):
    run([(7, 300), (130, 260)], scale=scale, max_new=max_new)


@pytest.mark.parametrize("max_new", [1, 1000])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", ["k", "v"])
def test_what_a_row_does_not_see(max_new, value, where):
    """A NaN or an infinity at one place: rows before it, or whose window is past it, have what they had; the others what the formula says."""
    from paper_2608_21614_b200 import attention
    seqs = [(150, 400), (1, 90)]
    for window in (0, 60):
        q, cache, batch, offsets = build(seqs, 8, 2, 64, 32, torch.bfloat16)
        batch.max_new = max_new
        att = attention.Attention(8, cache, window=window)
        before = att.attend(q, batch)[:151]
        c = getattr(cache, where)
        c[batch.table[0, 300 // 32].long(), 1, 300 % 32, 5] = value
        after = att.attend(q, batch)[:151]
        place = 250 + torch.arange(150, device="cuda")
        sees = (place >= 300) & ((place - 300 < window) if window else True)
        unseen = torch.cat((~sees, torch.ones(1, dtype=torch.bool, device="cuda")))
        u = torch.finfo(torch.bfloat16).eps / 2
        d = (after[unseen].double() - before[unseen].double()).abs()
        assert bool((d <= 4 * u * before[unseen].double().abs() + 2 * u).all())
        if where == "v" or math.isnan(value):
            check(after, None, q, cache, batch, seqs, offsets, True, window, 64 ** -0.5)


@pytest.mark.parametrize("max_new", [1, 1000])
def test_rows_that_are_nan_throughout(max_new):
    """Queries, keys or values of NaN from some place on: rows that see them are NaN, where the formula says so, the others as it says."""
    from paper_2608_21614_b200 import attention
    seqs = [(300, 700), (2, 90)]
    q, cache, batch, offsets = build(seqs, 8, 2, 64, 32, torch.bfloat16)
    batch.max_new = max_new
    att = attention.Attention(8, cache)
    q[40, 3] = math.nan
    q[41, 2, 7] = math.inf
    out = att.attend(q, batch)
    assert bool(torch.isnan(out[40, 3]).all()) and bool(torch.isnan(out[41, 2]).all())
    assert int(torch.isnan(out[:302]).any(-1).sum()) == 2
    q[40:42] = 1.0
    cache.v[batch.table[0, 500 // 32:(680 // 32) + 1].long(), :, :, :9] = math.nan
    out = att.attend(q, batch)
    check(out, None, q, cache, batch, seqs, offsets, True, 0, 0.125)


@pytest.mark.parametrize("max_new", [1, 1000])
def test_strides(max_new):
    """Queries as a part of a wider projection, results with heads before tokens."""
    from paper_2608_21614_b200 import attention
    seqs = [(1, 70), (33, 140), (5, 5)]
    q, cache, batch, offsets = build(seqs, 8, 4, 96, 16, torch.bfloat16, seed=3)
    batch.max_new = max_new
    wide = torch.randn(q.shape[0], 16, 96, device="cuda").bfloat16()
    wide[:, 4:12] = q
    out = torch.full((8, q.shape[0] + 3, 104), 9.0, dtype=torch.bfloat16, device="cuda")
    view = out.transpose(0, 1)[:q.shape[0], :, :96]
    att = attention.Attention(8, cache)
    att.attend(wide[:, 4:12], batch, out=view)
    check(view, None, q, cache, batch, seqs, offsets, True, 0, 96 ** -0.5)
    assert bool((out[:, q.shape[0]:] == 9).all()) and bool((out[:, :, 96:] == 9).all())


@pytest.mark.parametrize("max_new", [1, 1000])
def test_twice_the_same_bits_and_shared_workspace(max_new):
    from paper_2608_21614_b200 import attention
    q, cache, batch, _ = build([(5, 3000), (1, 200), (300, 2000)], 8, 2, 128, 64, torch.bfloat16)
    batch.max_new = max_new
    att = attention.Attention(8, cache)
    first = att.attend(q, batch)[:306]
    for _ in range(3):
        assert torch.equal(att.attend(q, batch)[:306], first)


@pytest.mark.parametrize("max_new", [1, 1000])
def test_pages_outside_the_cache(max_new):
    """They count as zeros and set the status word; other sequences are not touched."""
    from paper_2608_21614_b200 import attention, binding as B
    seqs = [(2, 200), (30, 100)]
    q, cache, batch, offsets = build(seqs, 4, 2, 64, 32, torch.bfloat16)
    batch.max_new = max_new
    att = attention.Attention(4, cache)
    want = att.attend(q, batch)[:32]
    for bad in (-1, cache.k.shape[0], 2 ** 31 - 1):
        batch.table[0, 1] = bad
        got = att.attend(q, batch)[:32]
        assert att.device_status() == B.SAEM_ERR_INVALID_ARG and att.device_status() == 0       # read and cleared
        assert torch.equal(got[2:], want[2:]) and bool(torch.isfinite(got[:2]).all())


def test_offsets_beyond_the_call_are_cut():
    """More rows in the offsets than the call has: nothing is written behind the tensors."""
    from paper_2608_21614_b200 import attention
    q, cache, batch, _ = build([(4, 50), (9, 60)], 4, 2, 64, 32, torch.bfloat16)
    for max_new in (1, 1000):
        batch.max_new = max_new
        for rows in (6, 12):
            out = torch.full((13, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
            attention.Attention(4, cache).attend(q[:rows], batch, out=out[:rows])
            assert bool((out[rows:] == 3).all()) and bool(torch.isfinite(out[:rows]).all())
    many, _, _, _ = build([(4, 50), (9, 60)], 64, 2, 64, 32, torch.bfloat16)
    out = torch.full((14, 64, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    attention.Attention(64, cache).attend(many[:13], batch, out=out[:13])                       # 832 rows: the form for many
    batch.offsets.copy_(torch.tensor([0, 20, 13], dtype=torch.int32))                           # and not ascending
    attention.Attention(64, cache).attend(many[:13], batch, out=out[:13])
    assert bool((out[13:] == 3).all()) and bool(torch.isfinite(out[:13]).all())


@pytest.mark.parametrize("max_new", [1, 1000])
def test_lengths_beyond_the_table_are_cut(max_new):
    from paper_2608_21614_b200 import attention
    seqs = [(3, 64)]
    q, cache, batch, offsets = build(seqs, 4, 2, 64, 32, torch.bfloat16, table_extra=0)
    batch.max_new = max_new
    batch.lengths.fill_(2 ** 31 - 1)
    out = attention.Attention(4, cache, causal=False).attend(q, batch)[:3]
    want = torch.stack([ref.attend(q[t:t + 1], *(ref.gather(c, batch.table[0], 64, 32) for c in (cache.k, cache.v)), 1, False, 0, 0.125)[0][0] for t in range(3)])
    assert bool(((out.double() - want).abs() < 0.05).all())


def test_more_places_than_32_bits_of_bytes():
    """A cache of more than 4 GB: the last pages are read where they are."""
    from paper_2608_21614_b200 import attention
    pages, heads, page, dim = 20000, 8, 128, 128                       # 5.2 GB of keys
    cache = attention.PagedCache.empty(pages, heads, page, dim)
    for c in (cache.k, cache.v):
        c[-4:] = torch.randn(4, heads, page, dim, generator=gen(4), device="cuda").bfloat16()
    q = torch.randn(60, 16, dim, generator=gen(5), device="cuda").bfloat16()                    # 27 rows behind the last sequence
    for max_new in (1, 1000):
        batch = attention.Batch(torch.tensor([0, 1, 33], dtype=torch.int32, device="cuda"), torch.tensor([300, 140], dtype=torch.int32, device="cuda"),
                                torch.tensor([[pages - 1, pages - 3, pages - 2], [pages - 2, pages - 4, 0]], dtype=torch.int32, device="cuda"), max_new)
        att = attention.Attention(16, cache)
        out = att.attend(q, batch)
        check(out, None, q, cache, batch, [(1, 300), (32, 140)], [0, 1, 33], True, 0, dim ** -0.5)


@pytest.mark.parametrize("tokens, max_new", [(528, 1), (800, 1000), (4096, 1000)])
def test_the_most_places(tokens, max_new):
    """2^31 - 2^16 places, of which every row's units alone nearly fill 32 bits with its neighbours': one page over and over, whose weights
    vanish beside those of another, which comes twice.  A chain of fp32 sums has at most 2^12 terms that count.  An item may take longer than the
    2 s that a wait has otherwise (4096 tokens)."""
    from paper_2608_21614_b200 import attention
    page, dim, entries = 65536, 8, 32767
    cache = attention.PagedCache.empty(2, 1, page, dim)
    for c in (cache.k, cache.v):
        c.copy_(torch.randn(c.shape, generator=gen(6), device="cuda"))
    cache.k[0] = -64.0                                              # scores below -180, and weights below 2^-200
    q = (torch.rand(tokens, 1, dim, generator=gen(7), device="cuda") + 1).bfloat16()
    table = torch.zeros(1, entries, dtype=torch.int32, device="cuda")
    table[0, [5000, 20000]] = 1
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    att = attention.Attention(1, cache)
    lse = torch.empty(tokens, 1, device="cuda")
    out = att.attend(q, attention.Batch(i32(0, tokens), i32(entries * page), table, max_new), lse=lse)
    assert att.device_status() == 0
    step = -(-tokens // 800)
    out, lse, q = out[::step], lse[::step], q[::step]
    want, size, want_lse, spread = ref.attend(q, cache.k[1], cache.v[1], len(q), False, 0, dim ** -0.5)
    delta = spread * ((dim + 8) * 2.0 ** -24 + 2.0 ** -22)
    bound = 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2 * delta[..., None] + 2.0 ** -11) * size
    assert float(((out.double() - want).abs() - bound).max()) <= 0
    want_lse += math.log(2)
    assert float(((lse.double() - want_lse).abs() - (2 * delta + 2.0 ** -11 + 2.0 ** -22 * want_lse.abs())).max()) <= 0


@pytest.mark.parametrize("max_new", [1, 1000])
def test_captured_and_replayed_while_lengths_grow(max_new):
    from paper_2608_21614_b200 import attention
    seqs = [(1, 500), (1, 64), (3, 900)]
    q, cache, batch, offsets = build(seqs, 8, 2, 128, 64, torch.bfloat16, garbage=0.5)
    batch.max_new = max_new
    att = attention.Attention(8, cache)
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        att.attend(q, batch, out=out)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            att.attend(q, batch, out=out)
    torch.cuda.current_stream().wait_stream(side)
    for grow in (0, 1, 7):
        batch.lengths += grow
        now = [(m, int(n)) for (m, _), n in zip(seqs, batch.lengths.tolist())]
        now = [(m, min(n, 8 * 64 if s == 0 else n)) for s, (m, n) in enumerate(now)]
        batch.lengths.copy_(torch.tensor([n for _, n in now], dtype=torch.int32))
        batch.table[1, 1] = 0
        graph.replay()
        torch.cuda.synchronize()
        check(out, None, q, cache, batch, now, offsets, True, 0, 128 ** -0.5)


def test_empty_calls():
    from paper_2608_21614_b200 import attention
    q, cache, batch, _ = build([(0, 10), (0, 0)], 4, 2, 64, 32, torch.bfloat16)
    att = attention.Attention(4, cache)
    assert att.attend(q[:0], batch).shape == (0, 4, 64)
    rows = torch.randn(3, 4, 64, device="cuda").bfloat16()
    out = torch.full_like(rows, 2.0)
    att.attend(rows, batch, out=out)
    assert bool((out == 2).all())
    none = attention.Batch(torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"),
                           torch.zeros(0, 4, dtype=torch.int32, device="cuda"))
    att.attend(rows, none, out=out)
    assert bool((out == 2).all())


def test_refusals_of_tensors():
    """What a kernel could not read is refused before it is launched: types, shapes, devices, strides, alignment."""
    from paper_2608_21614_b200 import attention, binding as B
    q, cache, batch, _ = build([(2, 30), (1, 20)], 4, 2, 64, 16, torch.bfloat16, spare_rows=0)
    att = attention.Attention(4, cache)

    def code(f):
        with pytest.raises(B.SaemError) as e:
            f()
        return e.value.code
    wide = torch.zeros(3, 4, 136, dtype=torch.bfloat16, device="cuda")
    flat = torch.zeros(3 * 4 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    assert code(lambda: att.attend(q.half(), batch)) == B.SAEM_ERR_INVALID_ARG
    assert code(lambda: att.attend(q.float(), batch)) == B.SAEM_ERR_INVALID_ARG
    assert code(lambda: att.attend(q[:, :2], batch)) == B.SAEM_ERR_SHAPE
    assert code(lambda: att.attend(q[..., :32], batch)) == B.SAEM_ERR_SHAPE
    assert code(lambda: att.attend(q.flatten(1), batch)) == B.SAEM_ERR_INVALID_ARG
    assert code(lambda: att.attend(q.cpu(), batch)) == B.SAEM_ERR_INVALID_ARG
    assert code(lambda: att.attend(wide[..., ::2][..., :64], batch)) == B.SAEM_ERR_INVALID_ARG
    assert code(lambda: att.attend(wide[..., 4:68], batch)) == B.SAEM_ERR_ALIGNMENT
    assert code(lambda: att.attend(flat[1:769].view(3, 4, 64), batch)) == B.SAEM_ERR_ALIGNMENT
    assert code(lambda: att.attend(q, batch, out=q[:2])) == B.SAEM_ERR_SHAPE
    assert code(lambda: att.attend(q, batch, out=torch.empty_like(q[:1]).expand(3, 4, 64))) == B.SAEM_ERR_SHAPE
    assert code(lambda: att.attend(q, batch, out=torch.empty_like(q, dtype=torch.float32))) == B.SAEM_ERR_INVALID_ARG
    for lse in (torch.empty(3, 4, device="cuda").half(), torch.empty(3, 4), torch.empty(4, 3, device="cuda").T):
        assert code(lambda: att.attend(q, batch, lse=lse)) == B.SAEM_ERR_INVALID_ARG
    assert code(lambda: att.attend(q, batch, lse=torch.empty(12, device="cuda"))) == B.SAEM_ERR_SHAPE
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    assert code(lambda: att.append(q, k[:2], k, batch)) == B.SAEM_ERR_SHAPE
    assert code(lambda: att.append(q, k, k.float(), batch)) == B.SAEM_ERR_INVALID_ARG
    assert code(lambda: att.append(q.float(), k, k, batch)) == B.SAEM_ERR_INVALID_ARG
    assert code(lambda: att.append(q, k, k, batch, q_out=torch.empty_like(q, dtype=torch.float16))) == B.SAEM_ERR_INVALID_ARG
    assert code(lambda: att.append(None, k, k, batch, positions=torch.zeros(2, dtype=torch.int32, device="cuda"))) == B.SAEM_ERR_SHAPE
    assert code(lambda: att.append(None, k, k, batch, positions=torch.zeros(3, dtype=torch.int64, device="cuda"))) == B.SAEM_ERR_INVALID_ARG
    assert code(lambda: attention.Attention(3, cache)) == B.SAEM_ERR_SHAPE
    assert code(lambda: attention.Attention(512, cache)) == B.SAEM_ERR_SHAPE
    assert code(lambda: attention.Attention(4, cache, window=-1)) == B.SAEM_ERR_SHAPE
    assert code(lambda: attention.Attention(4, cache, scale=0.0).attend(q, batch)) == B.SAEM_ERR_INVALID_ARG
    assert code(lambda: attention.PagedCache(cache.k, cache.v.half())) == B.SAEM_ERR_SHAPE
    assert code(lambda: attention.PagedCache(cache.k.float(), cache.v.float())) == B.SAEM_ERR_INVALID_ARG
    assert code(lambda: attention.PagedCache(cache.k[:, :, :8].contiguous(), cache.v[:, :, :8].contiguous())) == B.SAEM_ERR_SHAPE
    assert code(lambda: attention.PagedCache(cache.k.transpose(1, 2), cache.v.transpose(1, 2))) == B.SAEM_ERR_INVALID_ARG
    i = batch.lengths
    assert code(lambda: attention.Batch(batch.offsets, i.long(), batch.table)) == B.SAEM_ERR_INVALID_ARG
    assert code(lambda: attention.Batch(batch.offsets[:2], i, batch.table)) == B.SAEM_ERR_SHAPE
    assert code(lambda: attention.Batch(batch.offsets, i, batch.table[:1])) == B.SAEM_ERR_SHAPE
    assert code(lambda: attention.Batch(batch.offsets, i, batch.table.T.contiguous().T)) == B.SAEM_ERR_INVALID_ARG
    small = attention.Attention(4, cache)
    small.workspace = small.workspace[:8192]
    assert code(lambda: small.attend(q, batch)) == B.SAEM_ERR_WORKSPACE
    att.attend(q, batch)                                                        # and the handle still works
    assert att.device_status() == 0


@pytest.mark.parametrize("named_by", ["stream", "handle"])
def test_results_of_a_named_stream_keep_clear_of_the_current_one(named_by):
    from paper_2608_21614_b200 import attention, rotary
    seqs = [(64, 300), (1, 40)]
    q, cache, batch, _ = build(seqs, 8, 2, 64, 16, torch.bfloat16, garbage=0.0, spare_rows=0)
    k = torch.randn(65, 2, 64, device="cuda").bfloat16()
    turn = rotary.Rotary(64)
    att = attention.Attention(8, cache, rotary=turn)
    p = torch.arange(65, dtype=torch.int32, device="cuda")
    calls = {"append": lambda st: att.append(q, k, k, batch, stream=st), "attend": lambda st: att.attend(q, batch, stream=st), "rotate": lambda st: turn.rotate(q, p, stream=st)}
    for name, call in calls.items():
        want = call(None)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        torch.cuda.empty_cache()
        buf = torch.empty(q.shape, dtype=q.dtype, device="cuda")                # given back while the current stream will still write to it
        torch.cuda._sleep(40_000_000)
        buf.fill_(1)
        del buf
        got = call(side if named_by == "stream" else side.cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(got, want), name


def test_two_handles_on_two_streams_at_once():
    """Each with its own workspace: both as alone."""
    from paper_2608_21614_b200 import attention
    runs = []
    for seed, max_new in ((1, 1), (2, 1000)):
        q, cache, batch, _ = build([(3, 5000), (200, 2000), (1, 300)], 8, 2, 128, 64, torch.bfloat16, seed=seed, spare_rows=0)
        batch.max_new = max_new
        att = attention.Attention(8, cache)
        want = att.attend(q, batch)
        runs.append((att, q, batch, want, torch.empty_like(q), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(10):
        for att, q, batch, _, out, st in runs:
            att.attend(q, batch, out=out, stream=st)
    torch.cuda.synchronize()
    for att, _, _, want, out, _ in runs:
        assert torch.equal(out, want) and att.device_status() == 0
