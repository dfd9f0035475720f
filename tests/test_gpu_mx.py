"""The microscaled 4-bit operators on the GPU against plain 64-bit implementations (tests/mx_reference.py).

Quantisation, the way back and packing are exact.  A product's terms are exact too; its fp32 sum rounds once per MMA (64
terms), by at most one unit in the last place of what has been summed so far: |error| <= (k / 64 + 8) 2^-23 sum |a w|,
with 2^-8 of the result more for a bf16 output (half a unit of 8 significant bits).  The expert layer holds the
activations to 2^-13.8 of the largest of 32 neighbours; the tests allow 2^-12 of |Wd| |h|, doubled for the fp32 sums on the
way; what is below fp32's smallest numbers (2^-149 each, a sum of a few hundred of them) may vanish."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from paper_2608_21614_b200 import inputs as gen

pytestmark = pytest.mark.gpu
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def hard(rng, rows, cols):
    """Values with blocks of zeros, ties, subnormals, huge values, negative zeros and values that fall far below the block's."""
    x = rng.standard_normal((rows, cols)) * 10.0 ** rng.integers(-3, 4, (rows, (cols + 31) // 32)).repeat(32, 1)[:, :cols]
    x = x.astype(np.float32)
    flat = x.reshape(-1)
    for i, v in enumerate((0.0, -0.0, 6.0, 5.0, 2.5, -2.5, 0.25, 1e-38, 1e-42, 3e38, -0.1)):
        flat[i * 37 % flat.size] = v
    if cols >= 64:
        x[rows // 2, 32:64] = 0
    return x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,stride,offset", [
    (1, 1, 1, 0), (1, 32, 32, 0), (3, 31, 31, 0), (5, 33, 40, 0), (2, 64, 64, 1), (130, 128, 136, 8), (129, 1000, 1000, 0),
    (7, 999, 1003, 3), (257, 4104, 4104, 0), (1000, 8, 8, 0)])
def test_quantize_and_back(rows, cols, stride, offset, dtype):
    from paper_2608_21614_b200 import mx
    rng = np.random.default_rng(rows * 7919 + cols)
    flat = torch.zeros(offset + rows * stride, dtype=TORCH[dtype], device="cuda")
    x = flat[offset:].as_strided((rows, cols), (stride, 1), offset)
    x.copy_(torch.from_numpy(hard(rng, rows, cols)))
    q = mx.empty(rows, cols)
    q.codes.fill_(0xA5)
    q.scales.fill_(0xFF)
    mx.quantize(x, out=q)
    values, codes, scales = ref.quantize(f64(x))
    assert np.array_equal(q.codes.cpu().numpy().reshape(rows, -1), ref.pack_codes(codes))
    got = q.scales.cpu().numpy()
    assert np.array_equal(got[ref.scale_at(rows, scales.shape[1])], scales)
    n_block = scales.shape[1]
    padded = ref.scale_at(rows, (n_block + 3) // 4 * 4)[:, n_block:]
    assert not got[padded].any()                                        # blocks beyond the row: scale 2^-127, never NaN
    for out_type in TORCH.values():
        back = torch.full((offset + rows * stride,), 7.0, dtype=out_type, device="cuda")
        view = back.as_strided((rows, cols), (stride, 1), offset)
        mx.dequantize(q, out=view)
        assert np.array_equal(f64(view), values.astype(np.float32).astype(np.float64))
        if stride > cols and rows > 1:
            assert (back[offset + cols:offset + stride] == 7).all()     # nothing between the rows is written


def test_not_finite_blocks_become_nan():
    from paper_2608_21614_b200 import mx
    x = torch.randn(4, 96, device="cuda")
    x[0, 3], x[1, 40], x[2, 95] = float("inf"), float("nan"), float("-inf")
    back = f64(mx.dequantize(mx.quantize(x)))
    values = ref.quantize(f64(x))[0]
    assert np.array_equal(np.isnan(back), np.isnan(values)) and np.isnan(back).sum() == 96
    assert np.array_equal(back[~np.isnan(back)], values[~np.isnan(values)])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dequantize_every_code_and_scale(dtype):
    from paper_2608_21614_b200 import mx
    q = mx.empty(256, 32)
    codes = np.arange(32) % 16
    q.codes.copy_(torch.from_numpy(ref.pack_codes(np.tile(codes, (256, 1))).reshape(-1)))
    s = np.zeros(q.scales.numel(), np.uint8)
    s[ref.scale_at(256, 1)[:, 0]] = np.arange(256)
    q.scales.copy_(torch.from_numpy(s))
    got = f64(mx.dequantize(q, dtype=TORCH[dtype]))
    sign = np.where(codes & 8, -1.0, 1.0)
    with np.errstate(over="ignore"):
        want = (sign * ref.E2M1[codes & 7] * np.ldexp(1.0, np.arange(256) - 127)[:, None]).astype(np.float32).astype(np.float64)
    assert np.array_equal(got[:255], want[:255]) and np.isnan(got[255]).all()


# ------------------------------------------------------------------------------------------ products
def product_bound(a, w, out, k, bf16):
    bound = (k / 64 + 8) * 2.0 ** -23 * (np.abs(a) @ np.abs(w).T)
    return bound + (2.0 ** -8 * np.abs(out) * 1.01 if bf16 else 0)


def operands(m, n, k, seed):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.standard_normal((m, k)).astype(np.float32) * np.exp2(rng.integers(-6, 7, (m, 1))).astype(np.float32)).cuda()
    w = torch.from_numpy(rng.standard_normal((n, k)).astype(np.float32) * 0.1).cuda()
    return x, w, ref.quantize(f64(x))[0], ref.quantize(f64(w))[0]


SHAPES = [(1, 1, 1), (1, 128, 32), (1, 300, 4096), (2, 127, 31), (3, 129, 64), (8, 256, 96), (15, 64, 128), (16, 384, 160),
          (17, 130, 256), (33, 16, 288), (64, 1, 512), (100, 257, 1000), (127, 128, 2112), (128, 200, 320), (129, 128, 256),
          (200, 40, 96), (256, 256, 768), (257, 129, 64), (300, 384, 1500), (513, 130, 257), (1000, 640, 544), (1024, 1024, 1024),
          (2500, 1300, 416), (2304, 2300, 600), (4000, 1501, 136), (1025, 4096, 1024)]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product(m, n, k, out):
    from paper_2608_21614_b200 import mx
    x, w, a64, w64 = operands(m, n, k, m * 31 + n * 7 + k)
    qa, qw = mx.quantize(x), mx.quantize(w)
    buf = torch.full((m, n + 5), 3.0, dtype=TORCH[out], device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mx.matmul(qa, qw, out=buf[:, :n], status=status)
    want = a64 @ w64.T
    err = np.abs(f64(buf[:, :n]) - want)
    assert (err <= product_bound(a64, w64, want, k, out == "bf16")).all(), err.max()
    assert (buf[:, n:] == 3).all() and status.item() == 0               # nothing beside the result is written
    again = mx.matmul(qa, qw, dtype=TORCH[out])
    assert torch.equal(again, buf[:, :n])                               # a fixed order of sums


@pytest.mark.parametrize("x_type", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1, 200, 1000), (5, 128, 257), (40, 333, 96), (300, 140, 2048)])
def test_linear_is_quantize_then_product(m, n, k, x_type):
    from paper_2608_21614_b200 import mx
    x, w, _, _ = operands(m, n, k, m + n + k)
    wide = torch.zeros(m, k + 3, dtype=TORCH[x_type], device="cuda")
    xs = wide[:, 3:]                                                    # rows at no aligned address
    xs.copy_(x)
    qw = mx.quantize(w)
    linear = mx.Linear(qw, max_rows=m + 2)
    got = linear(xs, dtype=torch.float32)
    assert torch.equal(got, mx.matmul(mx.quantize(xs.contiguous()), qw, dtype=torch.float32))
    assert linear.device_status() == 0
    assert linear(xs[:0]).shape == (0, n)


def test_a_nan_block_reaches_its_row_or_column_only():
    from paper_2608_21614_b200 import mx
    x, w, a64, w64 = operands(40, 200, 320, 5)
    x[7, 100], w[131, 319] = float("nan"), float("inf")
    got = f64(mx.matmul(mx.quantize(x), mx.quantize(w), dtype=torch.float32))
    bad = np.zeros((40, 200), bool)
    bad[7], bad[:, 131] = True, True
    assert np.array_equal(np.isnan(got), bad)
    want = a64 @ w64.T
    assert (np.abs(got - want)[~bad] <= product_bound(a64, w64, want, 320, False)[~bad]).all()


def test_products_on_another_stream_and_in_a_graph():
    from paper_2608_21614_b200 import mx
    x, w, _, _ = operands(9, 256, 512, 3)
    linear = mx.Linear(mx.quantize(w), max_rows=9)
    want = linear(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert torch.equal(linear(x), want)
        out = torch.empty_like(want)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            linear(x, out=out)
        x.mul_(-2)
        graph.replay()
        side.synchronize()
    assert torch.equal(out, linear(x)) and not torch.equal(out, want)


def test_python_refusals():
    from paper_2608_21614_b200 import binding as B, mx
    x = torch.zeros(4, 64, device="cuda")
    q = mx.quantize(x)
    for call in (lambda: mx.quantize(x.half()), lambda: mx.quantize(x.t()), lambda: mx.quantize(x[0]), lambda: mx.quantize(x.cpu()),
                 lambda: mx.quantize(x, out=mx.empty(4, 65)), lambda: mx.dequantize(q, out=x[:3]), lambda: mx.matmul(q, mx.empty(3, 32)),
                 lambda: mx.matmul(q, q, out=x), lambda: mx.Linear(q, 2)(x), lambda: mx.Linear(q, 4)(x[:, :32])):
        with pytest.raises(B.SaemError):
            call()


# --------------------------------------------------------------------------------------- expert layer
def build(d, f, E, k, T, S=0, seed=0, pack="device", **kw):
    from paper_2608_21614_b200 import binding as B, mx
    from paper_2608_21614_b200.layer import MoELayer
    rng = np.random.default_rng(seed)
    layer = MoELayer(d, f, E, k, T, d_ff_shared=S * f, ffn_path=B.SAEM_FFN_MX, **kw)
    mats = [gen.expert_weights(rng, d, f) for _ in range(E + S)]
    exact = [[], [], []]
    for e, ms in enumerate(mats):
        wide = [torch.from_numpy(gen.bf16_bits_to_f32(m)) for m in ms]
        for i in range(3):
            exact[i].append(ref.quantize(wide[i].numpy())[0])
        if pack == "device":
            layer.load_expert_mx(0, e, e, *(mx.quantize(m.cuda().to(torch.bfloat16)) for m in wide))
        else:
            layer.load_expert(0, e, e, *ms)
    torch.cuda.synchronize()
    return layer, exact, rng


def check_step(layer, exact, logits, x, T, S=0, bf16=False):
    out = torch.full((T, layer.d), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    layer.step_fused_call(logits, x, T, out)
    order = np.argsort(-f64(logits), axis=-1, kind="stable")[:, :layer.k]
    top = np.take_along_axis(f64(logits), order, -1)
    w = np.exp(top - top.max(-1, keepdims=True))
    w /= w.sum(-1, keepdims=True)
    want, bound = ref.moe(f64(x), order, w, *exact, n_shared=S)
    limit = 2.0 ** -11 * bound + 2.0 ** -140 + (2.0 ** -8 * np.abs(want) * 1.01 if bf16 else 0)
    err = np.abs(f64(out) - want)
    assert (err <= limit).all(), (np.nanmax(err / limit), np.isnan(err).sum())
    assert layer.device_status() == 0
    return out


@pytest.mark.parametrize("d,f,E,k,T,S", [
    (128, 128, 1, 1, 1, 0), (256, 128, 4, 2, 1, 0), (128, 384, 8, 2, 3, 0), (512, 256, 16, 8, 1, 0), (512, 256, 16, 8, 8, 0),
    (640, 384, 8, 3, 7, 1), (256, 256, 6, 2, 9, 2), (384, 640, 5, 2, 17, 0), (256, 256, 3, 3, 33, 0), (1152, 128, 12, 4, 40, 0),
    (256, 512, 2, 1, 100, 1), (128, 256, 64, 6, 61, 2)])
def test_expert_layer(d, f, E, k, T, S):
    layer, exact, rng = build(d, f, E, k, T, S, seed=d + f + T)
    x = torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).cuda().to(torch.bfloat16)
    x[:, 3] *= 50
    logits = torch.from_numpy(rng.standard_normal((T, E)).astype(np.float32)).cuda()
    first = check_step(layer, exact, logits, x, T, S)
    again = torch.empty_like(first)
    layer.step_fused_call(logits, x, T, again)
    assert torch.equal(first, again)
    if T > 1:                                                           # fewer tokens than the context was made for
        check_step(layer, exact, logits[:1], x[:1], 1, S)
    layer.close()


def test_expert_layer_separate_calls_host_packing_and_bf16_out():
    from paper_2608_21614_b200 import binding as B
    layer, exact, rng = build(256, 256, 8, 2, 12, pack="host", out_dtype=B.SAEM_OUT_BF16)
    x = torch.from_numpy(rng.standard_normal((12, 256)).astype(np.float32)).cuda().to(torch.bfloat16)
    logits = torch.from_numpy(rng.standard_normal((12, 8)).astype(np.float32)).cuda()
    out = check_step(layer, exact, logits, x, 12, bf16=True)
    for T in (12, 5):
        stepwise = layer.step(logits, x, T)
        whole = torch.empty(T, 256, dtype=torch.bfloat16, device="cuda")
        layer.step_fused_call(logits, x, T, whole)
        # both hold h in 32 bits; the sums' order may differ between the forms
        assert np.abs(f64(stepwise.view(torch.bfloat16)) - f64(whole)).max() <= 2.0 ** -7 * np.abs(f64(whole)).max()
    host_out = torch.empty(12, 256, dtype=torch.bfloat16, pin_memory=True)
    layer.step_host(logits.cpu().pin_memory(), x.cpu().pin_memory(), 12, host_out)
    assert torch.equal(host_out, out.cpu())
    layer.close()


@pytest.mark.parametrize("T", [1, 6, 20])
def test_expert_layer_every_token_on_the_same_experts(T):
    layer, exact, rng = build(256, 384, 8, 2, T, seed=T)
    x = torch.from_numpy(rng.standard_normal((T, 256)).astype(np.float32)).cuda().to(torch.bfloat16)
    logits = torch.full((T, 8), -1.0, device="cuda")
    logits[:, 5], logits[:, 2] = 3.0, 2.0
    check_step(layer, exact, logits, x, T)
    layer.close()


@pytest.mark.parametrize("scale", [0.0, 1e-30, 1e-12, 1e12, 3e18])
def test_expert_layer_extreme_activations(scale):
    layer, exact, rng = build(256, 128, 4, 2, 4)
    x = torch.from_numpy((rng.standard_normal((4, 256)) * scale).astype(np.float32)).cuda().to(torch.bfloat16)
    logits = torch.from_numpy(rng.standard_normal((4, 4)).astype(np.float32)).cuda()
    if scale == 3e18:
        # the hidden activations, up to 1e38, still are finite in fp32; the sums with them may not be: compare what is
        out = torch.empty(4, 256, device="cuda")
        layer.step_fused_call(logits, x * 0.1, 4, out)
        assert torch.isfinite(out).all() and out.abs().max() > 1e30
    else:
        check_step(layer, exact, logits, x, 4)
    layer.close()


def test_a_token_that_is_not_finite_stays_alone():
    layer, exact, rng = build(256, 128, 4, 2, 6)
    x = torch.from_numpy(rng.standard_normal((6, 256)).astype(np.float32)).cuda().to(torch.bfloat16)
    logits = torch.zeros(6, 4, device="cuda")
    clean = check_step(layer, exact, logits, x, 6)
    x[2, 17] = float("nan")
    x[4, 200] = float("inf")
    out = torch.empty_like(clean)
    layer.step_fused_call(logits, x, 6, out)
    keep = [0, 1, 3, 5]
    assert torch.equal(out[keep], clean[keep]) and not torch.isfinite(out[2]).any() and not torch.isfinite(out[4]).any()
    layer.close()


@pytest.mark.parametrize("T", [2, 12])
def test_cache_calls_with_small_slots(T):
    from paper_2608_21614_b200 import binding as B, mx
    from paper_2608_21614_b200.layer import MoELayer
    d, f, E = 256, 256, 4
    rng = np.random.default_rng(1)
    mats = [gen.expert_weights(rng, d, f) for _ in range(E)]
    wide = [[gen.bf16_bits_to_f32(m) for m in ms] for ms in mats]
    exact = [[ref.quantize(wide[e][i])[0] for e in range(E)] for i in range(3)]
    layer = MoELayer(d, f, E, 2, T, slots_per_layer=2, temp_slots=1, ffn_path=B.SAEM_FFN_MX)
    h = layer.ctx.handle
    packed = []
    for e in (0, 1):
        q = [mx.quantize(torch.from_numpy(m).cuda()) for m in wide[e]]
        packed.append(layer.load_expert_mx(0, e, e, *q))
        host = layer.ctx.pack(*mats[e])
        torch.cuda.synchronize()
        assert torch.equal(packed[-1].cpu(), host)                      # the host's packing and the device's: the same bytes
    layer.copy_stream.synchronize()
    x = torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).cuda().to(torch.bfloat16)
    logits = torch.zeros(T, E, device="cuda")
    logits[:, :2] = 5.0
    check_step(layer, exact, logits, x, T)
    logits[0] = torch.tensor([0.0, 5.0, 0.0, 4.0], device="cuda")       # expert 3 has no slot
    out = torch.empty(T, d, device="cuda")
    layer.step_fused_call(logits, x, T, out)
    assert layer.device_status() == B.SAEM_ERR_NOT_RESIDENT
    layer.load_expert(0, 3, B.SAEM_TEMP, *mats[3])                      # through the temporary slot, from pinned memory
    check_step(layer, exact, logits, x, T)
    B.saem_cache_evict(h, 0, 0)
    layer.load_expert(0, 2, 0, *mats[2])
    logits[:] = torch.tensor([0.0, 5.0, 4.0, 0.0], device="cuda")
    check_step(layer, exact, logits, x, T)
    pinned = layer.ctx.pack(*mats[0])
    assert B.saem_cache_map_host(h, 0, 0, pinned, check=False) == B.SAEM_ERR_UNSUPPORTED
    with pytest.raises(B.SaemError):
        layer.load_expert_mx(0, 0, 0, mx.empty(f, d), mx.empty(f, d), mx.empty(f, d))
    layer.close()


@pytest.mark.parametrize("renorm", [0, 1])
@pytest.mark.parametrize("E,k,T", [(128, 8, 8), (97, 5, 3), (20, 8, 8), (8, 2, 7), (1, 1, 2), (33, 1, 8), (64, 6, 40), (16, 12, 20)])
def test_the_step_routes_as_saem_route_does(E, k, T, renorm):
    """Ties, zeros of both signs, infinities and NaN among the logits: the same experts, and the same weights to the bit."""
    from paper_2608_21614_b200 import binding as B, mx
    from paper_2608_21614_b200.layer import MoELayer
    rng = np.random.default_rng(E * k + T)
    layer = MoELayer(128, 128, E, k, T, ffn_path=B.SAEM_FFN_MX, renorm=renorm)
    q = [mx.quantize(torch.randn(128, 128, device="cuda")) for _ in range(3)]
    for e in range(E):
        layer.load_expert_mx(0, e, e, *q)
    logits = np.round(rng.standard_normal((T, E)) * 2).astype(np.float32) / 2
    odd = [0.0, -0.0, np.inf, -np.inf, np.nan, 1.0, 1.0]
    for t in range(T):
        logits[t, rng.integers(0, E, 3)] = rng.choice(odd, 3)
    logits[0] = -np.inf
    if T > 2:
        logits[1], logits[2] = np.nan, 0.0
    logits = torch.from_numpy(logits).cuda()
    x = torch.randn(T, 128, device="cuda").to(torch.bfloat16)
    out = torch.empty(T, 128, device="cuda")
    layer.step_fused_call(logits, x, T, out)
    idx = layer.ctx.step_tensor(0, (T, k), torch.int32).clone()
    w = layer.ctx.step_tensor(1, (T, k), torch.float32).clone()
    layer.route(logits, T)
    assert torch.equal(idx, layer.topk_idx[:T]) and torch.equal(w, layer.topk_w[:T])
    assert layer.device_status() == 0
    layer.close()


@pytest.mark.parametrize("E,k,T,S", [(16, 4, 9, 0), (64, 6, 33, 2), (128, 8, 64, 0), (20, 20, 51, 3), (1, 1, 64, 1), (128, 1, 32, 0)])
def test_the_step_indexes_as_saem_repack_does(E, k, T, S):
    from paper_2608_21614_b200 import binding as B, mx
    from paper_2608_21614_b200.layer import MoELayer
    layer = MoELayer(128, 128, E, k, T, d_ff_shared=128 * S, ffn_path=B.SAEM_FFN_MX)
    q = [mx.quantize(torch.randn(128, 128, device="cuda")) for _ in range(3)]
    for e in range(E + S):
        layer.load_expert_mx(0, e, e, *q)
    logits = torch.randn(T, E, device="cuda") + torch.linspace(0, 3, E, device="cuda")      # some experts stay empty
    x = torch.randn(T, 128, device="cuda").to(torch.bfloat16)
    layer.step_fused_call(logits, x, T, torch.empty(T, 128, device="cuda"))
    got = [layer.ctx.step_tensor(which, (n,), torch.int32).clone() for which, n in ((2, E + S), (3, E + S + 1), (4, T * k), (5, T * k))]
    layer.route(logits, T)
    layer.repack(x, T)
    for g, want in zip(got, (layer.counts, layer.offsets, layer.perm, layer.inv_perm)):
        assert torch.equal(g, want[:len(g)])
    assert layer.device_status() == 0
    layer.close()


def test_expert_ffn_of_one_expert_without_offsets():
    from paper_2608_21614_b200 import binding as B
    layer, exact, rng = build(256, 384, 1, 1, 70)
    x = torch.from_numpy(rng.standard_normal((70, 256)).astype(np.float32)).cuda().to(torch.bfloat16)
    for rows in (1, 8, 33, 70):
        y = torch.full((70, 256), 7.0, device="cuda")
        B.saem_expert_ffn(layer.ctx.handle, 0, x, None, rows, None, y)
        hid = ref.silu(f64(x)[:rows] @ exact[0][0].T) * (f64(x)[:rows] @ exact[1][0].T)
        assert (np.abs(f64(y)[:rows] - hid @ exact[2][0].T) <= 2.0 ** -11 * (np.abs(hid) @ np.abs(exact[2][0]).T)).all()
        assert (y[rows:] == 7).all()
    layer.close()


def test_all_rows_on_one_expert_of_many():
    """Segments far longer than the average that the row tiles are made for, and a long batch."""
    layer, exact, rng = build(128, 256, 32, 2, 300)
    x = torch.from_numpy(rng.standard_normal((300, 128)).astype(np.float32)).cuda().to(torch.bfloat16)
    logits = torch.from_numpy(rng.standard_normal((300, 32)).astype(np.float32)).cuda()
    logits[:, 7] += 20
    logits[:250, 30] += 10
    for T in (300, 129, 64, 11):
        check_step(layer, exact, logits[:T].contiguous(), x[:T].contiguous(), T)
    layer.close()


def test_subset_leaves_other_rows_alone():
    from paper_2608_21614_b200 import binding as B
    layer, exact, rng = build(256, 256, 4, 2, 10)
    x = torch.from_numpy(rng.standard_normal((10, 256)).astype(np.float32)).cuda().to(torch.bfloat16)
    layer.route(torch.from_numpy(rng.standard_normal((10, 4)).astype(np.float32)).cuda(), 10)
    layer.repack(x, 10)
    layer.y_packed.fill_(7.0)
    B.saem_expert_ffn(layer.ctx.handle, 0, layer.x_packed, layer.offsets, 20, [1, 2], layer.y_packed)
    off = layer.offsets.cpu().tolist()
    y, xp = f64(layer.y_packed), f64(layer.x_packed.view(torch.bfloat16))
    for e in range(4):
        rows = slice(off[e], off[e + 1])
        if e in (1, 2):
            hid = ref.silu(xp[rows] @ exact[0][e].T) * (xp[rows] @ exact[1][e].T)
            assert (np.abs(y[rows] - hid @ exact[2][e].T) <= 2.0 ** -11 * (np.abs(hid) @ np.abs(exact[2][e]).T)).all()
        else:
            assert (y[rows] == 7).all()
    layer.close()
