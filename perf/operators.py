"""What is measured of the 4-bit operators and the block norms, and their plain forms.

Four operators: the microscaled 4-bit format there and back ("mx"), a linear layer with 4-bit
weights and activations quantised on the way in ("linear"), a mixture-of-experts layer over 4-bit
experts for few tokens ("moe"), and the norms around a block with its gate and residual scale
("norm").  MXFP4: 32 consecutive elements of a row share one power of two, elements are E2M1.
"""
import math

import torch

own = False

BLOCK = 32
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
MX_BYTES = 17 / 32                       # per element: half a byte, and a scale byte for 32 of them


def listed():
    return [
        # an expert's matrix of a Mixtral-shaped layer, quantised when the checkpoint is loaded, and looked at again
        {"name": "mx-expert-matrix", "op": "mx", "rows": 14336, "cols": 4096, "dtype": "bf16"},
        # ragged activations in fp32: rows and columns that fill neither a tile nor a block
        {"name": "mx-ragged-f32", "op": "mx", "rows": 777, "cols": 2501, "dtype": "f32"},
        # one token through a dense projection while decoding
        {"name": "linear-1-token", "op": "linear", "m": 1, "n": 4096, "k": 4096, "dtype": "bf16", "out": "bf16"},
        # a decode batch through a wide projection
        {"name": "linear-16-tokens", "op": "linear", "m": 16, "n": 14336, "k": 4096, "dtype": "bf16", "out": "bf16"},
        # a short prompt, odd in every size, fp32 in and out (a head whose logits are kept in fp32)
        {"name": "linear-odd-f32", "op": "linear", "m": 333, "n": 2563, "k": 1500, "dtype": "f32", "out": "f32"},
        # prefill of a long prompt through a Mixtral-shaped projection
        {"name": "linear-prefill", "op": "linear", "m": 8192, "n": 14336, "k": 4096, "dtype": "bf16", "out": "bf16"},
        # one token through a layer of 128 small experts: the shortest decode step
        {"name": "moe-1-token", "op": "moe", "tokens": 1, "d": 2048, "f": 768, "experts": 128, "top_k": 8, "shared": 0},
        # a decode batch on the same layer
        {"name": "moe-8-tokens", "op": "moe", "tokens": 8, "d": 2048, "f": 768, "experts": 128, "top_k": 8, "shared": 0},
        # a decode batch on a layer of few wide experts
        {"name": "moe-wide-experts", "op": "moe", "tokens": 16, "d": 4096, "f": 14336, "experts": 8, "top_k": 2, "shared": 0},
        # an odd batch on a layer with always-on shared experts: the most tokens of this form
        {"name": "moe-shared-61-tokens", "op": "moe", "tokens": 61, "d": 2560, "f": 1536, "experts": 64, "top_k": 6, "shared": 2},
        # one token between two blocks while decoding
        {"name": "norm-1-token", "op": "norm", "tokens": 1, "d": 2048, "x": "bf16", "y": "f32", "gate": "none", "sigmoid": False, "post": True},
        # between two blocks in prefill: fp32 residual stream, a gate of each token
        {"name": "norm-prefill", "op": "norm", "tokens": 8192, "d": 4096, "x": "f32", "y": "bf16", "gate": "token", "sigmoid": True, "post": True},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["mx", "linear", "moe", "norm"])
    if op == "mx":
        return {"op": op, "rows": _spread(rng, 1, 14336), "cols": _spread(rng, 1, 4096), "dtype": rng.choice(["bf16", "f32"])}
    if op == "linear":
        return {"op": op, "m": _spread(rng, 1, 8192), "n": _spread(rng, 33, 14336), "k": _spread(rng, 31, 4096),
                "dtype": rng.choice(["bf16", "f32"]), "out": rng.choice(["bf16", "f32"])}
    if op == "moe":
        d, f = 128 * _spread(rng, 2, 32), 128 * _spread(rng, 1, 112)
        most = max(4, min(128, 8 * 4096 * 14336 // (d * f)))          # no more weights than the largest listed layer
        experts = _spread(rng, 4, most)
        shared = rng.choice([0, 0, 1, 2]) if experts + 2 <= most else 0
        return {"op": op, "tokens": _spread(rng, 1, 64), "d": d, "f": f, "experts": experts,
                "top_k": rng.randint(1, min(8, experts)), "shared": shared}
    return {"op": op, "tokens": _spread(rng, 1, 8192), "d": _spread(rng, 64, 4096), "x": rng.choice(["bf16", "f32"]),
            "y": rng.choice(["bf16", "f32"]), "gate": rng.choice(["none", "token", "channel", "full"]),
            "sigmoid": rng.random() < 0.5, "post": rng.random() < 0.75}


# ------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _activations(gen, rows, cols):
    """Unit normal with a few channels that are much larger, as activations have."""
    x = _normal(gen, rows, cols)
    loud = torch.rand(cols, generator=gen, device="cuda") < 0.01
    return x * torch.where(loud, 10.0, 1.0)


def _zipf(experts):
    p = [r ** -1.1 for r in range(1, experts + 1)]
    total = sum(p)
    return [v / total for v in p]


def _inputs(case, seed):
    """The numbers of a case, from the seed alone."""
    gen, op = _generator(seed), case["op"]
    if op == "mx":
        return {"x": _activations(gen, case["rows"], case["cols"]).to(DTYPES[case["dtype"]])}
    if op == "linear":
        return {"x": _activations(gen, case["m"], case["k"]).to(DTYPES[case["dtype"]]),
                "w": (_normal(gen, case["n"], case["k"]) * case["k"] ** -0.5).to(torch.bfloat16)}
    if op == "moe":
        d, f, total = case["d"], case["f"], case["experts"] + case["shared"]
        gumbel = -torch.log(-torch.log(torch.rand(case["tokens"], case["experts"], generator=gen, device="cuda").clamp(1e-12, 1 - 1e-7)))
        order = torch.randperm(case["experts"], generator=gen, device="cuda")
        logits = torch.log(torch.tensor(_zipf(case["experts"]), device="cuda"))[order] + gumbel
        return {"x": _activations(gen, case["tokens"], d).to(torch.bfloat16), "logits": logits,
                "gate": (_normal(gen, total, f, d) * d ** -0.5).to(torch.bfloat16),
                "up": (_normal(gen, total, f, d) * d ** -0.5).to(torch.bfloat16),
                "down": (_normal(gen, total, d, f) * f ** -0.5).to(torch.bfloat16)}
    t, d = case["tokens"], case["d"]
    gate = {"none": None, "token": (t, 1), "channel": (1, d), "full": (t, d)}[case["gate"]]
    return {"x": (3.0 * _activations(gen, t, d)).to(DTYPES[case["x"]]),
            "y": (0.5 * _activations(gen, t, d)).to(DTYPES[case["y"]]),
            "w_post": (1 + 0.1 * _normal(gen, d)).to(torch.bfloat16) if case["post"] else None,
            "w_pre": (1 + 0.1 * _normal(gen, d)).to(torch.bfloat16),
            "gate": None if gate is None else _normal(gen, *gate).to(torch.bfloat16)}


EPS, RESIDUAL_SCALE, BRANCH_SCALE = 1e-6, 0.75, 1.25


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    op = case["op"]
    # weights are quantised once, when a program loads them: each side keeps them in its own layout, and the
    # framework's side its buffers and its handle
    if not own:
        for name in {"linear": ("w",), "moe": ("gate", "up", "down")}.get(op, ()):
            state[name] = _quantize(state[name])
        return state
    if op == "norm":
        from paper_2608_21614_b200 import norms
        state["norm"] = norms.BlockNorm(case["d"], w_post=state["w_post"], w_pre=state["w_pre"], eps=EPS, residual_scale=RESIDUAL_SCALE,
                                        branch_scale=BRANCH_SCALE, gate=case["gate"], gate_sigmoid=case["sigmoid"])
        state["x_out"] = torch.empty_like(state["x"])
        state["n_out"] = torch.empty(state["x"].shape, dtype=torch.bfloat16, device="cuda")
        return state
    from paper_2608_21614_b200 import mx
    if op == "mx":
        state["packed"] = mx.empty(case["rows"], case["cols"])
        state["back"] = torch.empty_like(state["x"])
    elif op == "linear":
        state["linear"] = mx.Linear(mx.quantize(state.pop("w")), max_rows=case["m"])
        state["out"] = torch.empty(case["m"], case["n"], dtype=DTYPES[case["out"]], device="cuda")
    else:
        from paper_2608_21614_b200 import binding
        from paper_2608_21614_b200.layer import MoELayer
        layer = MoELayer(case["d"], case["f"], case["experts"], case["top_k"], case["tokens"], d_ff_shared=case["shared"] * case["f"],
                         ffn_path=binding.SAEM_FFN_MX, out_dtype=binding.SAEM_OUT_BF16)
        gate, up, down = (state.pop(n) for n in ("gate", "up", "down"))
        for e in range(case["experts"] + case["shared"]):
            layer.load_expert_mx(0, e, e, mx.quantize(gate[e]), mx.quantize(up[e]), mx.quantize(down[e]))
        torch.cuda.synchronize()
        state["layer"] = layer
        state["out"] = torch.empty(case["tokens"], case["d"], dtype=torch.bfloat16, device="cuda")
    return state


# ------------------------------------------------------------------------------------- plain forms
def _quantize(x):
    """MXFP4 of the rows of x [..., cols]: a code (sign, 3 bits) per element, two to a byte, and a scale byte per block."""
    cols = x.shape[-1]
    v = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK)).unflatten(-1, (-1, BLOCK))
    amax = v.abs().amax(-1, keepdim=True)
    e = ((amax.view(torch.int32) >> 23) - 129).clamp(min=-127)          # floor(log2 amax) - 2, from the exponent's bits
    a = v.abs() * ((127 - e) << 23).view(torch.float32)                # by 2^-e, exactly
    # to the nearest of E2M1, ties to the even mantissa
    code = (a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte() + (a > 5.0).byte()
    code = (code | (v < 0).byte() << 3).flatten(-2)
    return {"codes": code[..., 0::2] | code[..., 1::2] << 4, "scales": (e.squeeze(-1) + 127).byte(), "cols": cols}


def _dequantize(q):
    """The values that codes and scales stand for."""
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device="cuda")
    byte = torch.arange(256, device="cuda")
    pairs = torch.stack((table[byte & 15], table[byte >> 4]), -1)
    v = pairs[q["codes"].int()].flatten(-2).unflatten(-1, (-1, BLOCK))
    s = q["scales"].int()
    scale = torch.where(s > 0, s << 23, 1 << 22).view(torch.float32)    # 2^(s - 127): the exponent's bits, or the one subnormal
    return (v * scale.unsqueeze(-1)).flatten(-2)[..., :q["cols"]]


def _pick(q, experts):
    return {"codes": q["codes"][experts], "scales": q["scales"][experts], "cols": q["cols"]}


def _moe(state):
    case, x = state["case"], state["x"].float()
    tokens, experts, k, shared = case["tokens"], case["experts"], case["top_k"], case["shared"]
    value, index = torch.sort(state["logits"], dim=-1, descending=True, stable=True)
    value, index = value[:, :k], index[:, :k]
    weight = torch.exp(value - value[:, :1])
    weight = weight / weight.sum(-1, keepdim=True)
    if shared:                                                          # always on, with weight one
        index = torch.cat((index, torch.arange(experts, experts + shared, device="cuda").expand(tokens, shared)), -1)
        weight = torch.cat((weight, torch.ones(tokens, shared, device="cuda")), -1)
    if index.numel() < experts:                                         # few pairs: the weights of each pair's expert
        flat = index.flatten()
        rows = x.repeat_interleave(index.shape[1], 0).unsqueeze(-1)
        gate, up, down = (_dequantize(_pick(state[n], flat)) for n in ("gate", "up", "down"))
        g, u = gate @ rows, up @ rows
        y = (down @ (g / (1 + torch.exp(-g)) * u)).view(tokens, -1, case["d"])
        return (y * weight.unsqueeze(-1)).sum(1).to(torch.bfloat16)
    # more pairs: every expert on every token, then the weights of those that were chosen
    dense = torch.zeros(tokens, experts + shared, device="cuda").scatter(1, index, weight)
    g, u = x @ _dequantize(state["gate"]).mT, x @ _dequantize(state["up"]).mT
    y = (g / (1 + torch.exp(-g)) * u) @ _dequantize(state["down"]).mT
    return (y * dense.T.unsqueeze(-1)).sum(0).to(torch.bfloat16)


def _norm(state):
    case, y = state["case"], state["y"].float()
    if state["w_post"] is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS) * state["w_post"].float()
    if state["gate"] is not None:
        g = state["gate"].float()
        y = y * (1 / (1 + torch.exp(-g)) if case["sigmoid"] else g)
    x = RESIDUAL_SCALE * state["x"].float() + BRANCH_SCALE * y
    n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * state["w_pre"].float()
    return {"x": x.to(state["x"].dtype), "n": n.to(torch.bfloat16)}


def run(state):
    case, op = state["case"], state["case"]["op"]
    if own:
        if op == "mx":
            from paper_2608_21614_b200 import mx
            mx.quantize(state["x"], out=state["packed"])
            return mx.dequantize(state["packed"], out=state["back"])
        if op == "linear":
            return state["linear"](state["x"], out=state["out"])
        if op == "moe":
            state["layer"].step_fused_call(state["logits"], state["x"], case["tokens"], state["out"])
            return state["out"]
        state["norm"].leave(state["x"], state["y"], gate=state["gate"], x_out=state["x_out"], n_out=state["n_out"])
        return {"x": state["x_out"], "n": state["n_out"]}
    if op == "mx":
        return _dequantize(_quantize(state["x"])).to(state["x"].dtype)
    if op == "linear":
        return (_dequantize(_quantize(state["x"])) @ _dequantize(state["w"]).mT).to(DTYPES[case["out"]])
    return _moe(state) if op == "moe" else _norm(state)


# ------------------------------------------------------------------------------------------- work
def _active(case):
    """How many routed experts have a token, on average over draws of the routing."""
    import random
    rng, p = random.Random(7), [math.log(v) for v in _zipf(case["experts"])]
    total = 0
    for _ in range(4):
        seen = set()
        for _ in range(case["tokens"]):
            key = [v - math.log(-math.log(rng.uniform(1e-12, 1 - 1e-12))) for v in p]
            seen.update(sorted(range(len(p)), key=lambda e: -key[e])[:case["top_k"]])
        total += len(seen)
    return total / 4


def work(case):
    op = case["op"]
    if op == "mx":                                                      # there: read x, write packed; back: read packed, write x
        n = case["rows"] * case["cols"]
        return {"bytes": n * (2 * SIZE[case["dtype"]] + 2 * MX_BYTES), "flops": 4 * n}
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": n * k * MX_BYTES + m * k * SIZE[case["dtype"]] + m * n * SIZE[case["out"]], "flops": 2 * m * n * k}
    if op == "moe":
        t, d, f = case["tokens"], case["d"], case["f"]
        return {"bytes": (_active(case) + case["shared"]) * 3 * d * f * MX_BYTES + t * (4 * d + 4 * case["experts"]),
                "flops": 6 * t * (case["top_k"] + case["shared"]) * d * f}
    n, t, d = case["tokens"] * case["d"], case["tokens"], case["d"]
    gate = {"none": 0, "token": t, "channel": d, "full": n}[case["gate"]]
    return {"bytes": n * (2 * SIZE[case["x"]] + SIZE[case["y"]] + 2) + 2 * gate + 2 * d * (2 if case["post"] else 1), "flops": 12 * n}


# ----------------------------------------------------------------------------------- in 64 bits
def _exact_mx(x):
    """The nearest representable value of each element, searched for among the 15 of its block's scale."""
    cols = x.shape[-1]
    v = torch.nn.functional.pad(x.double(), (0, -cols % BLOCK)).unflatten(-1, (-1, BLOCK))
    top = v.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -125)
    step = top / torch.frexp(top)[0] / 8                                # 2^(floor(log2 top) - 2): top without its mantissa
    a = v.abs() / step
    # halves up to 2, wholes up to 4, twos above: torch.round goes to the even multiple, which is the even mantissa
    fine, middle, coarse = torch.round(2 * a) / 2, torch.round(a), 2 * torch.round(a / 2)
    out = torch.where(a <= 2, fine, torch.where(a <= 4, middle, coarse)).clamp(max=6) * step * torch.sign(v)
    return out.flatten(-2)[..., :cols]


def exact(case, seed):
    op, i = case["op"], _inputs(case, seed)
    if op == "mx":
        return _exact_mx(i["x"])
    if op == "linear":
        return _exact_mx(i["x"]) @ _exact_mx(i["w"]).T
    if op == "moe":
        x, out = i["x"].double(), torch.zeros(case["tokens"], case["d"], dtype=torch.float64, device="cuda")
        value, index = torch.topk(i["logits"].double(), case["top_k"])
        weight = torch.softmax(value, -1)
        for e in range(case["experts"] + case["shared"]):
            if e < case["experts"]:
                token, slot = torch.nonzero(index == e, as_tuple=True)
                w = weight[token, slot]
            else:
                token, w = torch.arange(case["tokens"], device="cuda"), torch.ones(case["tokens"], dtype=torch.float64, device="cuda")
            if len(token) == 0:
                continue
            g, u, down = x[token] @ _exact_mx(i["gate"][e]).T, x[token] @ _exact_mx(i["up"][e]).T, _exact_mx(i["down"][e])
            out.index_add_(0, token, w[:, None] * ((g * torch.sigmoid(g) * u) @ down.T))
        return out
    x, y = i["x"].double(), i["y"].double()
    if i["w_post"] is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * i["w_post"].double()
    if i["gate"] is not None:
        y = y * (torch.sigmoid(i["gate"].double()) if case["sigmoid"] else i["gate"].double())
    x = RESIDUAL_SCALE * x + BRANCH_SCALE * y
    return {"x": x, "n": x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * i["w_pre"].double()}
