"""CPU checks of the attention operators: refusals before anything is enqueued, frequencies, and their fixed-point form."""
import ctypes
import math
from fractions import Fraction

import pytest
import torch

from paper_2608_21614_b200 import binding as B

P = 4096                                                                        # an address that is never read


def rot(**kw):
    c = dict(head_dim=128, rotary_dim=64, interleaved=0, eps=1e-6, amplitude=1.0)
    c.update(kw)
    return B.saem_rotary_config(**c)


def test_rotate_refusals():
    def call(x=P, w=P, turns=P, positions=P, out=P, r=None, cfg=True, **kw):
        c = dict(rotary=rot(**(r or {})), x_dtype=1, out_dtype=1, w_dtype=1, heads=4, tokens=3, x_token_stride=512, x_head_stride=128, out_token_stride=512,
                 out_head_stride=128)
        c.update(kw)
        return B.saem_rotate(B.saem_rotate_config(**c) if cfg else None, x, w, turns, positions, out, stream=0, check=False)
    assert call(cfg=False) == call(x=None) == call(out=None) == call(positions=None) == call(turns=None) == B.SAEM_ERR_INVALID_ARG
    assert call(x_dtype=3) == call(out_dtype=-1) == call(w_dtype=2) == call(r=dict(eps=-1.0)) == call(r=dict(eps=math.nan)) == B.SAEM_ERR_INVALID_ARG
    assert call(r=dict(amplitude=math.inf)) == B.SAEM_ERR_INVALID_ARG
    for d, rd in ((0, 0), (4, 0), (132, 8), (136, 8), (-8, 0), (64, 72), (64, 12), (64, -8)):
        assert call(r=dict(head_dim=d, rotary_dim=rd)) == B.SAEM_ERR_SHAPE
    assert call(tokens=-1) == call(heads=0) == call(tokens=2 ** 30, heads=3) == call(x_token_stride=-1) == call(x_head_stride=-1) == B.SAEM_ERR_SHAPE
    assert call(out_head_stride=127) == call(out_token_stride=511) == call(out_token_stride=0) == B.SAEM_ERR_SHAPE
    assert call(out_token_stride=100, out_head_stride=400) == B.SAEM_ERR_SHAPE                 # heads before tokens, which overlap
    assert call(x=P + 1) == call(out=P + 1) == call(w=P + 1) == call(turns=P + 4) == call(positions=P + 2) == B.SAEM_ERR_ALIGNMENT
    assert call(tokens=0, x=None, out=None, positions=None) == B.SAEM_OK


def cache(**kw):
    c = dict(k=P, v=P, pages=10, page_size=64, kv_heads=2, head_dim=128, dtype=1)
    c.update(kw)
    return B.saem_kv_cache(**c)


def batch(**kw):
    c = dict(offsets=P, lengths=P, table=P, table_stride=4, seqs=2, tokens=5, max_pages=4, max_new=3)
    c.update(kw)
    return B.saem_batch(**c)


BAD_CACHES = [(dict(dtype=0), B.SAEM_ERR_INVALID_ARG), (dict(k=None), B.SAEM_ERR_INVALID_ARG), (dict(v=None), B.SAEM_ERR_INVALID_ARG), (dict(page_size=8), B.SAEM_ERR_SHAPE),
              (dict(page_size=24), B.SAEM_ERR_SHAPE), (dict(page_size=65552), B.SAEM_ERR_SHAPE), (dict(pages=0), B.SAEM_ERR_SHAPE), (dict(kv_heads=0), B.SAEM_ERR_SHAPE),
              (dict(head_dim=136), B.SAEM_ERR_SHAPE), (dict(head_dim=100), B.SAEM_ERR_SHAPE), (dict(pages=2 ** 31 // 128), B.SAEM_ERR_SHAPE),
              (dict(pages=2 ** 40), B.SAEM_ERR_SHAPE), (dict(k=P + 8), B.SAEM_ERR_ALIGNMENT), (dict(v=P + 2), B.SAEM_ERR_ALIGNMENT)]
BAD_BATCHES = [(dict(offsets=None), B.SAEM_ERR_INVALID_ARG), (dict(lengths=None), B.SAEM_ERR_INVALID_ARG), (dict(table=None), B.SAEM_ERR_INVALID_ARG),
               (dict(seqs=-1), B.SAEM_ERR_SHAPE), (dict(seqs=65537), B.SAEM_ERR_SHAPE), (dict(tokens=-1), B.SAEM_ERR_SHAPE), (dict(max_pages=-1), B.SAEM_ERR_SHAPE),
               (dict(table_stride=3), B.SAEM_ERR_SHAPE), (dict(max_new=-1), B.SAEM_ERR_SHAPE), (dict(offsets=P + 2), B.SAEM_ERR_ALIGNMENT),
               (dict(table=P + 1), B.SAEM_ERR_ALIGNMENT)]


def test_append_refusals():
    def call(q=P, k=P, v=P, w_q=P, w_k=P, turns=P, positions=None, q_out=P, status=P, c=None, b=None, r=None, **kw):
        cfg = dict(rotary=rot(**(r or {})), q_heads=4, x_dtype=0, w_dtype=0, q_token_stride=1024, q_head_stride=128, k_token_stride=1024, k_head_stride=128,
                   v_token_stride=1024, v_head_stride=128, out_token_stride=512, out_head_stride=128)
        cfg.update(kw)
        return B.saem_kv_append(B.saem_append_config(**cfg), c or cache(), b or batch(), q, k, v, w_q, w_k, turns, positions, q_out, status, stream=0, check=False)
    for bad, code in BAD_CACHES:
        assert call(c=cache(**bad)) == code, bad
    for bad, code in BAD_BATCHES:
        assert call(b=batch(**bad)) == code, bad
    assert call(k=None) == call(v=None) == call(q_out=None) == call(q=None) == call(turns=None) == B.SAEM_ERR_INVALID_ARG
    assert call(q=None, q_out=None) == call(x_dtype=4) == call(w_dtype=2) == call(r=dict(eps=-1e-6)) == B.SAEM_ERR_INVALID_ARG     # w_q without q
    assert call(r=dict(head_dim=64)) == call(q_heads=0) == call(k_token_stride=-1) == call(v_head_stride=-1) == call(q_token_stride=-8) == B.SAEM_ERR_SHAPE
    assert call(out_token_stride=511) == call(out_head_stride=64) == call(q_heads=2 ** 30) == B.SAEM_ERR_SHAPE
    assert call(k=P + 2) == call(q=P + 1) == call(w_q=P + 2) == call(turns=P + 4) == call(positions=P + 1) == call(status=P + 2) == call(q_out=P + 1) == B.SAEM_ERR_ALIGNMENT
    assert call(b=batch(tokens=0, offsets=None), k=None) == call(b=batch(seqs=0, lengths=None), q=None) == B.SAEM_OK
    assert B.saem_kv_append(None, cache(), batch(), P, P, P, P, P, P, None, P, stream=0, check=False) == B.SAEM_ERR_INVALID_ARG
    assert B.saem_kv_append(B.saem_append_config(), None, batch(), P, P, P, P, P, P, None, P, stream=0, check=False) == B.SAEM_ERR_INVALID_ARG


def test_attend_refusals():
    def call(q=P, out=P, lse=None, ws=P, size=1 << 40, c=None, b=None, **kw):
        cfg = dict(q_heads=8, causal=1, window=0, scale=0.1, q_token_stride=1024, q_head_stride=128, out_token_stride=1024, out_head_stride=128)
        cfg.update(kw)
        return B.saem_attend(B.saem_attend_config(**cfg), c or cache(), b or batch(), q, out, lse, ws, size, stream=0, check=False)
    for bad, code in BAD_CACHES:
        assert call(c=cache(**bad)) == code, bad
    for bad, code in BAD_BATCHES:
        assert call(b=batch(**bad)) == code, bad
    assert call(q=None) == call(out=None) == call(ws=None) == call(scale=0.0) == call(scale=-1.0) == call(scale=math.nan) == call(scale=math.inf) == B.SAEM_ERR_INVALID_ARG
    assert call(q_heads=0) == call(q_heads=7) == call(q_heads=258) == call(window=-1) == B.SAEM_ERR_SHAPE
    assert call(q_token_stride=-8) == call(out_token_stride=1016) == call(out_head_stride=120) == call(b=batch(tokens=2 ** 30)) == B.SAEM_ERR_SHAPE
    assert call(q=P + 8) == call(out=P + 2) == call(lse=P + 2) == call(ws=P + 512) == call(q_token_stride=1028) == call(out_token_stride=1028) == B.SAEM_ERR_ALIGNMENT
    assert call(b=batch(tokens=0), q=None) == call(b=batch(seqs=0, offsets=None), ws=None) == B.SAEM_OK
    assert B.saem_attend(None, cache(), batch(), P, P, None, P, 1, stream=0, check=False) == B.SAEM_ERR_INVALID_ARG
    assert B.saem_attend_workspace_bytes(None) == 0 and B.saem_attend_workspace_bytes(cache(page_size=1)) == 0


def test_struct_sizes():
    assert ctypes.sizeof(B.saem_rotary_config) == 20 and ctypes.sizeof(B.saem_rotate_config) == 80
    assert ctypes.sizeof(B.saem_kv_cache) == 40 and ctypes.sizeof(B.saem_batch) == 48
    assert ctypes.sizeof(B.saem_append_config) == 96 and ctypes.sizeof(B.saem_attend_config) == 48


def test_tensors_on_the_host_are_refused():
    from paper_2608_21614_b200 import attention, rotary
    with pytest.raises(B.SaemError) as e:
        attention.PagedCache.empty(2, 2, 16, 64, device="cpu")
    assert e.value.code == B.SAEM_ERR_INVALID_ARG
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(B.SaemError):
        attention.Batch(i, i[:1], i.view(1, 2))
    r = rotary.Rotary(64, device="cpu")
    x = torch.zeros(2, 3, 64)
    with pytest.raises(B.SaemError):
        r.rotate(x, i)
    from paper_2608_21614_b200.mx import _calls
    assert _calls.attend(bytes(B.saem_attend_config()), x, x, x, i, i, i, 1, x, None, x, None) == B.SAEM_ERR_INVALID_ARG
    assert _calls.append(bytes(B.saem_append_config()), None, x, x, None, None, None, None, x, x, i, i, i, 1, None, None, None) == B.SAEM_ERR_INVALID_ARG
    with pytest.raises(TypeError):
        _calls.rotate(b"", x, None, None, i, x, None)
    with pytest.raises(TypeError):
        _calls.attend(bytes(B.saem_attend_config()))


def test_rotary_arguments():
    from paper_2608_21614_b200 import rotary
    for a, kw in (((132,), {}), ((0,), {}), ((64, 12), {}), ((64, 72), {}), ((64,), dict(radians=[0.1] * 31))):
        with pytest.raises(B.SaemError) as e:
            rotary.Rotary(*a, device="cpu", **kw)
        assert e.value.code == B.SAEM_ERR_SHAPE
    for kw in (dict(base=-1.0), dict(amplitude=math.inf), dict(radians=[math.nan] * 32), dict(scaling={"kind": "linear"}), dict(scaling={"kind": "other", "factor": 2}),
               dict(scaling={"kind": "linear", "factor": 0.5}), dict(scaling={"kind": "linear", "factor": 2, "more": 1}), dict(scaling={"factor": 2}),
               dict(scaling={"kind": "bands", "factor": 2, "original": 4096, "low": 4, "high": 1}), dict(scaling={"kind": "yarn", "factor": 2}),
               dict(scaling={"kind": "yarn", "factor": 2, "original": 4096, "beta_fast": 1, "beta_slow": 32})):
        with pytest.raises(B.SaemError) as e:
            rotary.Rotary(64, device="cpu", **kw)
        assert e.value.code == B.SAEM_ERR_INVALID_ARG, kw


def test_frequencies():
    from paper_2608_21614_b200.rotary import frequencies
    plain, one = frequencies(64, 10000.0)
    assert one == 1.0 and plain[0] == 1.0 and plain[31] == pytest.approx(10000.0 ** (-62 / 64), rel=1e-15) and len(plain) == 32
    assert frequencies(0) == ([], 1.0)
    linear, _ = frequencies(64, scaling={"kind": "linear", "factor": 4.0})
    assert all(a == b / 4 for a, b in zip(linear, plain))
    base, _ = frequencies(64, scaling={"kind": "base", "factor": 8.0})
    assert base[0] == 1.0 and base[31] == pytest.approx(plain[31] / 8, rel=1e-12)
    bands, _ = frequencies(64, scaling={"kind": "bands", "factor": 8.0, "original": 4096.0, "low": 1.0, "high": 4.0})
    for f, g in zip(plain, bands):
        turns = 4096 * f / (2 * math.pi)
        assert g == f if turns >= 4 else g == f / 8 if turns <= 1 else f / 8 < g < f
    assert any(f / 8 < g < f for f, g in zip(plain, bands))
    yarn, amplitude = frequencies(64, scaling={"kind": "yarn", "factor": 32.0, "original": 4096.0})
    assert amplitude == pytest.approx(0.1 * math.log(32) + 1)
    # the pair that turns beta times within the original context: index dim ln(original / (2 pi beta)) / (2 ln base)
    at = lambda beta: 64 * math.log(4096 / (2 * math.pi * beta)) / (2 * math.log(10000.0))      # noqa: E731
    first, last = math.floor(at(32)), math.ceil(at(1))
    for i, (f, g) in enumerate(zip(plain, yarn)):
        r = min(1.0, max(0.0, (i - first) / (last - first)))
        assert g == pytest.approx(f * (1 - r) + f / 32 * r, rel=1e-14)
    assert yarn[0] == plain[0] and yarn[31] == pytest.approx(plain[31] / 32, rel=1e-14)
    assert frequencies(64, scaling={"kind": "yarn", "factor": 2.0, "original": 4096.0, "amplitude": 3.0})[1] == 3.0


def test_turns_are_exact_to_their_last_bit():
    from paper_2608_21614_b200.rotary import turns
    two_pi = Fraction(628318530717958647692528676655900576839433879875021, 10 ** 50)
    for f in (1.0, 0.5, 1e-4, 12345.678, -0.25, 0.0, 2 * math.pi):
        got = turns([f])[0]
        assert -2 ** 63 <= got < 2 ** 63
        exact = Fraction(f) / two_pi * 2 ** 64
        off = (Fraction(got) - exact) % 2 ** 64
        assert min(off, 2 ** 64 - off) <= Fraction(1, 2) + Fraction(1, 2 ** 30)
        # a far position: the angle that the integer product stands for
        p = 2 ** 31 - 1
        angle = ((got * p) % 2 ** 64) / 2 ** 64 * 2 * math.pi
        want = float((Fraction(f) * p / two_pi) % 1) * 2 * math.pi
        assert min(abs(angle - want), 2 * math.pi - abs(angle - want)) < 1e-8
