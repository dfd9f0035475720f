"""Attention at the edges of what a call may hold: lengths that the table cuts.

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
