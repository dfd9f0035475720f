"""Attention at the edges of what a call may hold: lengths that the table cuts, values that are not finite, weights that are small beside
another, and what weights lose to 16 bits.

Bounds as in test_gpu_attention.py: a weight's rounding u and the result's u, 2 delta for the scores, 2^-18 for exponentials and sums."""
import math

import pytest
import torch

import test_gpu_attention as base

pytestmark = pytest.mark.gpu


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def formula(q, k, v, seen, scale):
    """q [n, heads, dim], k and v [kv_heads, places, dim], seen [n, places]: (out, size, delta) in 64 bits."""
    q, k, v = q.double(), *(x.double().repeat_interleave(q.shape[1] // x.shape[0], 0) for x in (k, v))
    s = torch.where(seen, scale * torch.einsum("thd,hjd->htj", q, k), -math.inf)
    p = torch.softmax(torch.where(seen.any(1)[:, None], s, 0.0), 2) * seen
    spread = torch.where(seen, scale * torch.einsum("thd,hjd->htj", q.abs(), k.abs()), 0.0).amax(2).T
    return (p @ v).transpose(0, 1), (p @ v.abs()).transpose(0, 1), spread * ((q.shape[2] + 8) * 2.0 ** -24 + 2.0 ** -22)


def within(got, want, size, delta):
    u = torch.finfo(got.dtype).eps / 2
    return bool(((got.double() - want).abs() <= u * want.abs() + (u + 2 * delta[..., None] + 2.0 ** -18) * size).all())


@pytest.mark.parametrize("max_new", [1, 1000])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 20), (False, 0), (False, 20), (True, 300)])
@pytest.mark.parametrize("extra_seqs", [0, 40])
def test_lengths_beyond_the_table_leave_tokens_at_their_places(max_new, causal, window, extra_seqs):
    """A token's place goes by the length alone, also where the table has fewer places (the others are not seen): 10 tokens behind the table, 150 on
    both sides of its end.  The status word says so, and neighbours are as without them."""
    from paper_2608_21614_b200 import attention, binding as B
    page, dim, hq, hk = 32, 64, 8, 2
    news, lengths = [10, 150, 3] + [1] * extra_seqs, [100, 260, 90] + [5] * extra_seqs
    g = base.gen(1)
    cache = attention.PagedCache(*(torch.randn(11, hk, page, dim, generator=g, device="cuda").bfloat16() for _ in range(2)))
    rows = [[4, 2], [0, 5, 7, 1, 9, 3], [8, 6, 10]] + [[10]] * extra_seqs
    att = attention.Attention(hq, cache, causal=causal, window=window)
    offsets = [sum(news[:s]) for s in range(len(news) + 1)]
    q = torch.randn(offsets[-1] + 101, hq, dim, generator=g, device="cuda").bfloat16()          # more than 768 rows in all: max_new chooses the form
    for s in (0, 1):                                                                            # one table of two entries, one of six
        table = torch.full((len(news), len(rows[s])), 10, dtype=torch.int32, device="cuda")
        for r, pages in enumerate(rows):
            table[r, :len(pages)] = torch.tensor(pages[:len(rows[s])], dtype=torch.int32)
        out, lse = torch.empty_like(q), torch.full(q.shape[:2], 7.0, device="cuda")
        cut = [n if r == s else min(n, len(rows[s]) * page) for r, n in enumerate(lengths)]     # the other sequences within the table
        att.attend(q, attention.Batch(i32(*offsets), i32(*cut), table, max_new), out=out, lse=lse)
        assert att.device_status() == B.SAEM_ERR_INVALID_ARG and att.device_status() == 0
        for r in (s, 2):
            t, n = slice(offsets[r], offsets[r + 1]), news[r]
            k, v = (c[table[r].long()].transpose(0, 1).flatten(1, 2) for c in (cache.k, cache.v))
            place, j = cut[r] - n + torch.arange(n, device="cuda")[:, None], torch.arange(k.shape[1], device="cuda")
            seen = (j < cut[r]) & ((j <= place) if causal else (place == place)) & ((j > place - window) if window else (j >= 0))
            want, size, delta = formula(q[t], k, v, seen, dim ** -0.5)
            assert within(out[t], want, size, delta), (s, r)
            none = ~seen.any(1)
            assert bool((out[t][none] == 0).all()) and bool((lse[t][none] == -math.inf).all())


def test_a_sequence_without_new_tokens_may_have_any_length():
    from paper_2608_21614_b200 import attention
    cache = attention.PagedCache(*(torch.randn(4, 2, 16, 64, generator=base.gen(2), device="cuda").bfloat16() for _ in range(2)))
    q = torch.randn(200, 8, 64, generator=base.gen(3), device="cuda").bfloat16()
    att = attention.Attention(8, cache)
    for max_new in (1, 1000):
        att.attend(q, attention.Batch(i32(0, 0, 2, 2), i32(1000, 20, 2 ** 31 - 1), i32(0, 1, 2, 3, 0, 0).view(3, 2), max_new))
        assert att.device_status() == 0


@pytest.mark.parametrize("max_new", [1, 1000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 60), (False, 0), (False, 60)])
@pytest.mark.parametrize("extra_seqs", [0, 40])
def test_values_that_are_not_finite_here_and_there(max_new, dtype, causal, window, extra_seqs):
    """NaN and infinities of both signs, a few in every column of some pages and many in some columns: each result is NaN, infinite or finite as the
    formula says, whatever else its tile holds."""
    from paper_2608_21614_b200 import attention
    seqs = [(150, 400), (1, 90), (300, 2000), (2, 700)] + [(1, 40)] * extra_seqs
    q, cache, batch, offsets = base.build(seqs, 8, 2, 80, 32, dtype, seed=5)
    batch.max_new = max_new
    g = base.gen(6)
    odd = torch.tensor([math.nan, math.inf, -math.inf], device="cuda").to(dtype)
    for s, (n, length) in enumerate(seqs):
        many = 12 if s < 4 else 1
        r = lambda top, k: torch.randint(0, top, (k,), generator=g, device="cuda")                              # noqa: E731
        place = torch.cat((r(length, many), length - 1 - r(min(n, length), many)))              # anywhere, and where some of the tokens are
        column = torch.cat((r(80, many), r(4, many)))
        cache.v[batch.table[s, place // 32].long(), r(2, 2 * many), place % 32, column] = odd[r(3, 2 * many)]
    att = attention.Attention(8, cache, causal=causal, window=window)
    out = att.attend(q, batch)
    assert att.device_status() == 0
    base.check(out, None, q, cache, batch, seqs, offsets, causal, window, 80 ** -0.5)


@pytest.mark.parametrize("max_new", [1, 1000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_value_that_is_not_finite_at_the_end_of_half_a_million_places(max_new, dtype):
    """The last token of the first sequence alone sees it; summing the others again takes longer than a wait within the kernel may, and the sequences
    behind have to be there all the same.  At most 3 pages of 256 places have weights that count: 2^-14 for the sums of so many."""
    from paper_2608_21614_b200 import attention
    page, dim, hq, hk, n, entries = 256, 64, 8, 2, 20, 2048
    g = base.gen(8)
    cache = attention.PagedCache(*(torch.randn(5, hk, page, dim, generator=g, device="cuda").to(dtype) for _ in range(2)))
    cache.k[0] = -16.0                                              # scores below -128 and below all others by far more than 100
    cache.k[1:] *= 0.1
    q = (torch.rand(8 * n + 20, hq, dim, generator=g, device="cuda") + 1).to(dtype)
    table = torch.zeros(8, entries, dtype=torch.int32, device="cuda")
    table[:, 700], table[:, 1500], table[:, -1], table[0, -1] = 1, 2, 3, 4
    cache.v[4, :, -1, 5], cache.v[4, 1, -1, 6] = math.nan, math.inf
    att = attention.Attention(hq, cache)
    out = att.attend(q, attention.Batch(i32(*range(0, 8 * n + 1, n)), i32(*[entries * page] * 8), table, max_new))
    assert att.device_status() == 0
    u = torch.finfo(dtype).eps / 2
    for s in range(8):
        k, v = (c[[1, 2, 4 if s == 0 else 3]].transpose(0, 1).flatten(1, 2) for c in (cache.k, cache.v))
        seen = torch.arange(3 * page, device="cuda") <= 3 * page - n + torch.arange(n, device="cuda")[:, None]
        want, size, delta = formula(q[s * n:(s + 1) * n], k, torch.nan_to_num(v, 0.0, 0.0, 0.0), seen, dim ** -0.5)
        got = out[s * n:(s + 1) * n]
        if s == 0:
            assert bool(torch.isnan(got[-1, :, 5]).all()) and bool((got[-1, 4:, 6] == math.inf).all())
            got = got.clone()
            got[-1, :, 5], got[-1, 4:, 6] = want[-1, :, 5].to(dtype), want[-1, 4:, 6].to(dtype)
        assert bool(((got.double() - want).abs() <= u * want.abs() + (u + 2 * delta[..., None] + 2.0 ** -14) * size).all()), s


@pytest.mark.parametrize("dtype,new,length", [(torch.bfloat16, 1, 131072), (torch.bfloat16, 2048, 2048), (torch.float16, 1, 131072), (torch.float16, 2048, 2048)])
def test_a_nan_that_is_seen_does_not_make_a_call_slow(dtype, new, length):
    """Such a result is NaN and needs no second sum: of the rows' own places at most one more look at the values is paid for.  At the last place of
    2048 tokens, the 63 tokens x 4 heads before it in their item do not see it and are summed again: 32 rows a warp, 128 steps of 16 places,
    each below 2 us, which are 8.2 ms."""
    from paper_2608_21614_b200 import attention
    cache = attention.PagedCache(*(torch.randn(length // 64, 8, 64, 128, generator=base.gen(s), device="cuda").to(dtype) for s in (1, 2)))
    q = torch.randn(new, 32, 128, generator=base.gen(3), device="cuda").to(dtype)
    batch = attention.Batch(i32(0, new), i32(length), torch.arange(length // 64, dtype=torch.int32, device="cuda")[None], new)
    att, out = attention.Attention(32, cache), torch.empty_like(q)

    def best():
        times = []
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            att.attend(q, batch, out=out)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)
    plain = best()
    for place in (0, length // 2, length - 1):
        kept = cache.v[place // 64, :, place % 64, 3].clone()
        cache.v[place // 64, :, place % 64, 3] = math.nan
        slow = best()
        assert bool(torch.isnan(out[-1, :, 3]).all()) and bool(torch.isfinite(out[-1, :, 4:]).all())
        cache.v[place // 64, :, place % 64, 3] = kept
        print("%s %d over %d, NaN at %d: %.3f ms, without %.3f ms" % (dtype, new, length, place, slow, plain))
        again = 32 * 128 * 2e-3 if new > 1 and place == length - 1 else 0.0
        assert slow < 30 * plain + again                            # summing all again took 400 to 900 times as long


@pytest.mark.parametrize("max_new", [1, 1000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [14.3, 20.608, 25.15])
def test_many_small_weights_beside_a_large_one(max_new, dtype, bits):
    """A million places whose weights are 2^-bits of a few whose values are zero, in as many sequences as leave each to one CTA, whose warps (four, or
    two groups) all have one of the few.  A float16 weight's last bit is 2^-24 of 2^7 times the largest at least: 2^(bits - 32) of a small one.
    Sums: a warp's 2^14 products of 16 places lose 2^-23 each (a group's 2^15 do, of sums half as large), 2^16 additions to a weight of 1 at most 2^-24 each."""
    from paper_2608_21614_b200 import attention
    page, dim, entries, seqs = 256, 64, 4096, 296
    k, v = torch.zeros(8, 1, page, dim, device="cuda"), torch.rand(8, 1, page, dim, generator=base.gen(9), device="cuda") + 0.5
    few = torch.tensor([0, 16, 32, 48, 128], device="cuda")
    k[0, 0, few, 0], v[0, 0, few] = bits * math.log(2), 0.0
    cache = attention.PagedCache(k.to(dtype), v.to(dtype))
    q = torch.zeros(seqs, 4, dim, device="cuda", dtype=dtype)
    q[..., 0] = 8.0                                                 # scores: the keys' first elements
    table = 1 + torch.arange(entries, dtype=torch.int32, device="cuda")[None].repeat(seqs, 1) % 7
    table[:, 0] = 0
    att = attention.Attention(4, cache, causal=False)
    lse = torch.empty(seqs, 4, device="cuda")
    out = att.attend(q, attention.Batch(i32(*range(seqs + 1)), i32(*[entries * page] * seqs), table, max_new), lse=lse)
    times = torch.bincount(table[0], minlength=8).double().repeat_interleave(page)
    score = cache.k[:, 0].flatten(0, 1)[:, 0].double()
    p = torch.softmax(score + times.log(), 0)
    want = p @ cache.v[:, 0].flatten(0, 1).double()                 # values are positive
    u, sums = torch.finfo(dtype).eps / 2, 2.0 ** -8 + 2.0 ** -9 + 2.0 ** -18
    assert att.device_status() == 0
    assert float((out.double() / want - 1).abs().max()) <= 2 * u + sums + (2.0 ** (bits - 32) if dtype == torch.float16 else 0.0)
    assert float((lse.double() - torch.logsumexp(score + times.log(), 0)).abs().max()) <= sums


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("q_heads,kv_heads,dim", [(8, 1, 128), (16, 4, 64), (3, 3, 96)])
@pytest.mark.parametrize("length", [3, 40, 700, 20000])
def test_weights_of_up_to_eight_rows_lose_little_to_16_bits(dtype, q_heads, kv_heads, dim, length):
    """A weight is the sum of two 16-bit ones, of which the first is below it by 2^-7 of it at most and the second off by 2^-9 of itself: 2^-16."""
    from paper_2608_21614_b200 import attention
    seqs = [(1, length)] * 3 + [(8 // (q_heads // kv_heads), length)]
    q, cache, batch, offsets = base.build(seqs, q_heads, kv_heads, dim, 32, dtype, seed=12, spare_rows=0)
    out = attention.Attention(q_heads, cache).attend(q, batch)
    u = torch.finfo(dtype).eps / 2
    for s, (n, _) in enumerate(seqs):
        t = slice(offsets[s], offsets[s + 1])
        k, v = (base.ref.gather(c, batch.table[s], length, 32) for c in (cache.k, cache.v))
        want, size, _, spread = base.ref.attend(q[t], k, v, n, True, 0, dim ** -0.5)
        delta = spread * ((dim + 8) * 2.0 ** -24 + 2.0 ** -22)
        off = (out[t].double() - want).abs() - u * want.abs() - (2.0 ** -16 + 2 * delta[..., None] + 2.0 ** -18) * size
        assert float(off.max()) <= torch.finfo(dtype).tiny * 2


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_infinities_that_few_rows_see(dtype, value):
    """Times a weight and times what the weight lost to 16 bits: the infinity, also where a weight is exact or very small."""
    from paper_2608_21614_b200 import attention
    k, v = (torch.zeros(40, 1, 32, 64, device="cuda", dtype=dtype) for _ in range(2))
    q = torch.zeros(3, 2, 64, device="cuda", dtype=dtype)
    q[:, :, 0] = 8.0
    k[:, :, :, 0] = -torch.randint(0, 30, (40, 1, 32), generator=base.gen(1), device="cuda").to(dtype) / 2              # weights from 1 to e^-14.5
    v[7, 0, 3, 5], v[20, 0, 31, 6], v[39, 0, 31, 7] = value, value, value
    k[7, 0, 3, 0], k[20, 0, 31, 0] = 0.0, -60.0
    batch = attention.Batch(i32(0, 1, 3), i32(1280, 1280), torch.arange(40, dtype=torch.int32, device="cuda").repeat(2, 1))
    out = attention.Attention(2, attention.PagedCache(k, v)).attend(q, batch).float()
    want = torch.zeros(3, 2, 64, device="cuda")
    want[:, :, 5:7], want[[0, 2], :, 7] = value, value                       # the last place is the last token's
    assert torch.equal(torch.nan_to_num(out, 3.0, 1.0, 2.0), torch.nan_to_num(want, 3.0, 1.0, 2.0))
