"""What is measured of the attention operators, and their plain forms.

Three operators: the norm of each head with the rotation of its positions ("rotate"), the same on the way of new queries, keys
and values, the keys and values appended to a paged cache ("append"), and attention of the new tokens over that cache
("attend").  Pages hold [kv_heads, page, head_dim]; a table names each sequence's pages in order; a sequence's length counts its
new tokens, which are its last ones.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS, BASE, ORIGINAL = 1e-6, 10000.0, 4096.0


def listed():
    return [
        # the heads of one token's queries while decoding
        {"name": "rotate-1-token", "op": "rotate", "tokens": 1, "heads": 32, "dim": 128, "rot": 128, "interleaved": False, "norm": True,
         "x": "bf16", "out": "bf16", "factor": 1.0},
        # queries and keys of a prompt, far into a long context, pairs next to each other
        {"name": "rotate-prefill", "op": "rotate", "tokens": 8192, "heads": 40, "dim": 128, "rot": 128, "interleaved": True, "norm": True,
         "x": "bf16", "out": "bf16", "factor": 32.0},
        # a decode batch: one token of each of 16 sequences, in a layer of 32 query and 4 key heads
        {"name": "append-decode", "op": "append", "seqs": 16, "new": 1, "ctx": 2048, "ragged": True, "q_heads": 32, "kv_heads": 4, "dim": 128,
         "rot": 128, "interleaved": False, "norm": True, "page": 64, "x": "bf16", "cache": "bf16", "factor": 1.0},
        # an odd chunk in fp32, a part of each head rotated, small pages
        {"name": "append-chunk-f32", "op": "append", "seqs": 3, "new": 777, "ctx": 3001, "ragged": True, "q_heads": 20, "kv_heads": 5, "dim": 96,
         "rot": 48, "interleaved": True, "norm": False, "page": 16, "x": "f32", "cache": "f16", "factor": 8.0},
        # a long prompt's tokens into the cache
        {"name": "append-prefill", "op": "append", "seqs": 1, "new": 8192, "ctx": 8192, "ragged": False, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "rot": 128, "interleaved": False, "norm": True, "page": 64, "x": "bf16", "cache": "bf16", "factor": 1.0},
        # the shortest call: one token after a short prompt
        {"name": "attend-1-token", "op": "attend", "seqs": 1, "new": 1, "ctx": 1000, "ragged": False, "q_heads": 32, "kv_heads": 4, "dim": 128,
         "page": 64, "cache": "bf16", "causal": True, "window": 0},
        # one token at the end of a long chain of thought
        {"name": "attend-1-token-long", "op": "attend", "seqs": 1, "new": 1, "ctx": 131072, "ragged": False, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "page": 64, "cache": "bf16", "causal": True, "window": 0},
        # a decode batch of sequences of very different lengths
        {"name": "attend-decode-ragged", "op": "attend", "seqs": 16, "new": 1, "ctx": 16384, "ragged": True, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "page": 16, "cache": "bf16", "causal": True, "window": 0},
        # a few tokens each, checked at once, in a sliding window; odd heads
        {"name": "attend-few-window", "op": "attend", "seqs": 7, "new": 5, "ctx": 5003, "ragged": True, "q_heads": 20, "kv_heads": 5, "dim": 96,
         "page": 32, "cache": "f16", "causal": True, "window": 2000},
        # a chunk of a prompt over what is in the cache already
        {"name": "attend-chunk", "op": "attend", "seqs": 1, "new": 512, "ctx": 16384, "ragged": False, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "page": 64, "cache": "bf16", "causal": True, "window": 0},
        # prompts of several lengths beside decoding sequences, small heads
        {"name": "attend-mixed", "op": "attend", "seqs": 9, "new": 1025, "ctx": 4099, "ragged": True, "q_heads": 12, "kv_heads": 12, "dim": 64,
         "page": 128, "cache": "bf16", "causal": True, "window": 0},
        # prefill of a long prompt
        {"name": "attend-prefill", "op": "attend", "seqs": 1, "new": 8192, "ctx": 8192, "ragged": False, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "page": 64, "cache": "bf16", "causal": True, "window": 0},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "append", "attend", "attend"])
    dim = rng.choice([64, 80, 96, 112, 128, 128])
    kv_heads, group = rng.choice([1, 2, 3, 4]), rng.choice([1, 2, 3, 4, 6, 8])
    turn = {"rot": rng.choice([dim, dim, 8 * rng.randint(1, dim // 8)]), "interleaved": rng.random() < 0.5, "norm": rng.random() < 0.7,
            "factor": rng.choice([1.0, 4.0, 32.0])}
    if op == "rotate":
        return {"op": op, "tokens": _spread(rng, 1, 8192), "heads": rng.randint(1, 40), "dim": dim, **turn,
                "x": rng.choice(["bf16", "f16", "f32"]), "out": rng.choice(["bf16", "f16"])}
    page, cache = rng.choice([16, 32, 64, 128, 256]), rng.choice(["bf16", "bf16", "f16"])
    if op == "append":
        seqs = _spread(rng, 1, 64)
        new = _spread(rng, 1, max(1, 8192 // seqs))
        return {"op": op, "seqs": seqs, "new": new, "ctx": new + _spread(rng, 1, max(2, 32768 // seqs)) - 1, "ragged": rng.random() < 0.7,
                "q_heads": kv_heads * group, "kv_heads": kv_heads, "dim": dim, **turn, "page": page, "x": rng.choice(["bf16", "f16", "f32"]),
                "cache": cache}
    # as much as the largest listed prefill at most: queries x keys, and keys
    seqs = _spread(rng, 1, 64)
    ctx = _spread(rng, 1, max(2, 131072 // seqs))
    most = max(1, min(ctx, 8192 * 8192 // (seqs * ctx)))
    new = rng.choice([1, 1, min(ctx, rng.randint(2, 8)), _spread(rng, 1, most)])
    return {"op": op, "seqs": seqs, "new": min(new, most), "ctx": ctx, "ragged": rng.random() < 0.7, "q_heads": kv_heads * group,
            "kv_heads": kv_heads, "dim": dim, "page": page, "cache": cache, "causal": rng.random() < 0.85,
            "window": rng.choice([0, 0, _spread(rng, 1, ctx + 1)])}


# ------------------------------------------------------------------------------------------- inputs
def _sequences(case):
    """(new tokens, length) of each sequence: the first one's are the case's, the others' spread below them."""
    rng, news, lengths = random.Random(case["seqs"] * 7919 + case["ctx"]), [], []
    for s in range(case["seqs"]):
        whole = s == 0 or not case["ragged"]
        news.append(case["new"] if whole else _spread(rng, 1, case["new"]))
        lengths.append(case["ctx"] if whole else max(news[-1], _spread(rng, 1, case["ctx"])))
    return news, lengths


def _frequencies(case):
    """Radians per position of each pair, in 64 bits: slow pairs of a context grown by `factor` turn that much slower, fast ones
    as before, and those between by a mean of the two."""
    f = [BASE ** (-2.0 * i / case["rot"]) for i in range(case["rot"] // 2)]
    if case["factor"] == 1.0:
        return f
    low, high = 1.0, 4.0                                # turns within the original context
    def mixed(v):
        share = min(1.0, max(0.0, (ORIGINAL * v / (2 * math.pi) - low) / (high - low)))
        return v * (share + (1 - share) / case["factor"])
    return [mixed(v) for v in f]


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _heads(gen, tokens, heads, dim, dtype):
    """Heads out of a projection: unit normal with a few channels that are larger."""
    loud = torch.rand(heads, dim, generator=gen, device="cuda") < 0.02
    return (_normal(gen, tokens, heads, dim) * torch.where(loud, 5.0, 1.0)).to(DTYPES[dtype])


def _inputs(case, seed):
    """The numbers of a case, from the seed alone."""
    gen, op, dim = _generator(seed), case["op"], case["dim"]
    if op == "rotate":
        start = int(torch.randint(0, int(ORIGINAL * case["factor"]), (1,), generator=gen, device="cuda"))
        return {"x": _heads(gen, case["tokens"], case["heads"], dim, case["x"]),
                "w": (1 + 0.1 * _normal(gen, dim)).to(torch.bfloat16) if case["norm"] else None,
                "positions": torch.arange(start, start + case["tokens"], dtype=torch.int32, device="cuda")}
    news, lengths = _sequences(case)
    per = -(-max(lengths) // case["page"])
    pages = sum(-(-n // case["page"]) for n in lengths)
    order, table, at = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32), torch.zeros(case["seqs"], per, dtype=torch.int32, device="cuda"), 0
    for s, n in enumerate(lengths):
        k = -(-n // case["page"])
        table[s, :k] = order[at:at + k]
        at += k
    tokens = sum(news)
    i = {"offsets": torch.tensor([sum(news[:s]) for s in range(case["seqs"] + 1)], dtype=torch.int32, device="cuda"),
         "lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda"), "table": table}
    shape, dtype = (pages, case["kv_heads"], case["page"], dim), DTYPES[case["cache"]]
    if op == "append":
        # out of one projection, one after the other
        all_heads = _heads(gen, tokens, case["q_heads"] + 2 * case["kv_heads"], dim, case["x"])
        i["q"], i["k"], i["v"] = all_heads.split([case["q_heads"], case["kv_heads"], case["kv_heads"]], 1)
        for name in ("w_q", "w_k"):
            i[name] = (1 + 0.1 * _normal(gen, dim)).to(torch.bfloat16) if case["norm"] else None
        i["cache_k"], i["cache_v"] = torch.zeros(shape, dtype=dtype, device="cuda"), torch.zeros(shape, dtype=dtype, device="cuda")
        return i
    # a direction that queries share and that the first key of each sequence has most of: it draws weight from everywhere
    sink = _normal(gen, dim)
    i["q"] = (_normal(gen, tokens, case["q_heads"], dim) + 0.5 * sink).to(dtype)
    i["cache_k"], i["cache_v"] = _normal(gen, *shape).to(dtype), _normal(gen, *shape).to(dtype)
    i["cache_k"][table[:, 0].long(), :, 0] = sink.to(dtype)
    return i


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    op, dim = case["op"], case["dim"]
    if not own:
        if op != "attend":
            state["frequencies"] = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
        return state
    from paper_2608_21614_b200 import attention, rotary
    if op != "attend":
        scaling = None if case["factor"] == 1.0 else {"kind": "bands", "factor": case["factor"], "original": ORIGINAL, "low": 1.0, "high": 4.0}
        state["rotary"] = rotary.Rotary(dim, rotary_dim=case["rot"], base=BASE, interleaved=case["interleaved"], scaling=scaling)
    if op == "rotate":
        state["out"] = torch.empty(state["x"].shape, dtype=DTYPES[case["out"]], device="cuda")
        return state
    cache = attention.PagedCache(state["cache_k"], state["cache_v"])
    state["batch"] = attention.Batch(state["offsets"], state["lengths"], state["table"], max_new=case["new"])
    state["out"] = torch.empty(state["q"].shape, dtype=DTYPES[case["cache"]], device="cuda")
    if op == "append":
        state["attention"] = attention.Attention(case["q_heads"], cache, rotary=state["rotary"], w_q=state["w_q"], w_k=state["w_k"], eps=EPS)
    else:
        state["attention"] = attention.Attention(case["q_heads"], cache, causal=case["causal"], window=case["window"])
    return state


# ------------------------------------------------------------------------------------- plain forms
def _norm_and_rotate(case, x, w, angle):
    """x [T, heads, dim], angle [T, rot / 2] in 64 bits; 32 bits out."""
    x = x.float()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    rot = case["rot"]
    cos, sin = torch.cos(angle).float().unsqueeze(1), torch.sin(angle).float().unsqueeze(1)
    turned, rest = x[..., :rot], x[..., rot:]
    if case["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = turned[..., :rot // 2], turned[..., rot // 2:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, rest), -1)


def _places(state, tokens):
    """Of each token: its sequence and its place there."""
    offsets, t = state["offsets"].long(), torch.arange(tokens, device="cuda")
    seq = (t.unsqueeze(1) >= offsets[1:]).sum(1)
    return seq, state["lengths"].long()[seq] - offsets[seq + 1] + t


def _append(state):
    case, dtype = state["case"], DTYPES[state["case"]["cache"]]
    seq, place = _places(state, state["q"].shape[0])
    angle = place.double().unsqueeze(1) * state["frequencies"]
    page, slot = state["table"].long()[seq, place // case["page"]], place % case["page"]
    q = _norm_and_rotate(case, state["q"], state["w_q"], angle).to(dtype)
    state["cache_k"][page, :, slot] = _norm_and_rotate(case, state["k"], state["w_k"], angle).to(dtype)
    state["cache_v"][page, :, slot] = state["v"].to(dtype)
    return {"q": q, "k": state["cache_k"], "v": state["cache_v"]}


def _attend(state):
    case, q = state["case"], state["q"].float()
    tokens, group, dim = q.shape[0], case["q_heads"] // case["kv_heads"], case["dim"]
    seq, place = _places(state, tokens)
    # queries in rows of their own for each sequence, keys and values in the order of their positions
    row = torch.arange(tokens, device="cuda") - state["offsets"].long()[seq]
    padded = torch.zeros(case["seqs"], case["new"], case["kv_heads"], group, dim, device="cuda")
    padded[seq, row] = q.view(tokens, case["kv_heads"], group, dim)
    at = torch.full((case["seqs"], case["new"]), -1, device="cuda")
    at[seq, row] = place
    k, v = (state[n][state["table"].long()].transpose(1, 2).flatten(2, 3).float() for n in ("cache_k", "cache_v"))
    j = torch.arange(k.shape[2], device="cuda")
    seen = j < state["lengths"].long().view(-1, 1, 1)
    if case["causal"]:
        seen = seen & (j <= at.unsqueeze(2))
    if case["window"]:
        seen = seen & (j > at.unsqueeze(2) - case["window"])
    seen = seen.expand(-1, case["new"], -1).repeat_interleave(group, 1).unsqueeze(1)
    scores = padded.permute(0, 2, 1, 3, 4).flatten(2, 3) @ k.mT * dim ** -0.5
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-1e30)                # rows that see nothing: weights of zero
    weights = torch.exp_(scores.sub_(top))
    total = weights.sum(-1, keepdim=True)
    out = (weights @ v) / torch.where(total > 0, total, 1.0)
    return out.unflatten(2, (case["new"], group)).permute(0, 2, 1, 3, 4)[seq, row].reshape(tokens, case["q_heads"], dim).to(DTYPES[case["cache"]])


def run(state):
    case, op = state["case"], state["case"]["op"]
    if own:
        if op == "rotate":
            return state["rotary"].rotate(state["x"], state["positions"], weight=state["w"], eps=EPS, out=state["out"])
        if op == "append":
            q = state["attention"].append(state["q"], state["k"], state["v"], state["batch"], q_out=state["out"])
            return {"q": q, "k": state["cache_k"], "v": state["cache_v"]}
        return state["attention"].attend(state["q"], state["batch"], out=state["out"])
    if op == "rotate":
        angle = state["positions"].double().unsqueeze(1) * state["frequencies"]
        return _norm_and_rotate(case, state["x"], state["w"], angle).to(DTYPES[case["out"]])
    return _append(state) if op == "append" else _attend(state)


# ------------------------------------------------------------------------------------------- work
def work(case):
    dim = case["dim"]
    if case["op"] == "rotate":
        n = case["tokens"] * case["heads"] * dim
        return {"bytes": n * (SIZE[case["x"]] + SIZE[case["out"]]) + 4 * case["tokens"], "flops": 10 * n}
    news, lengths = _sequences(case)
    tokens = sum(news)
    if case["op"] == "append":
        n = tokens * (case["q_heads"] + 2 * case["kv_heads"]) * dim
        return {"bytes": n * (SIZE[case["x"]] + SIZE[case["cache"]]) + 4 * tokens, "flops": 10 * n}
    keys = pairs = 0
    for new, length in zip(news, lengths):
        first = length - new
        window = case["window"] or length + 1
        keys += length - max(0, first - window + 1)
        if case["causal"]:
            whole = min(new, max(0, window - first))                    # tokens whose window reaches the beginning
            pairs += whole * first + whole * (whole + 1) // 2 + (new - whole) * window
        else:
            pairs += sum(length - max(0, p - window + 1) for p in range(first, length))
    return {"bytes": 2 * SIZE[case["cache"]] * dim * (tokens * case["q_heads"] + keys * case["kv_heads"]), "flops": 4 * dim * case["q_heads"] * pairs}


# ----------------------------------------------------------------------------------- in 64 bits
def _exact_rotation(case, x, w, positions):
    """Pairs as complex numbers, turned by e^(i p f)."""
    x = x.double()
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.double()
    rot, p = case["rot"], positions.double()
    phase = torch.polar(torch.ones(len(p), rot // 2, dtype=torch.float64, device="cuda"),
                        torch.outer(p, torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")))[:, None]
    out = x.clone()
    if case["interleaved"]:
        out[..., :rot] = torch.view_as_real(torch.view_as_complex(x[..., :rot].unflatten(-1, (-1, 2)).contiguous()) * phase).flatten(-2)
    else:
        z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * phase
        out[..., :rot // 2], out[..., rot // 2:rot] = z.real, z.imag
    return out


def exact(case, seed):
    i, op = _inputs(case, seed), case["op"]
    if op == "rotate":
        return _exact_rotation(case, i["x"], i["w"], i["positions"])
    news, lengths = _sequences(case)
    if op == "append":
        positions = torch.cat([torch.arange(n - m, n, device="cuda") for m, n in zip(news, lengths)])
        q, k, v = _exact_rotation(case, i["q"], i["w_q"], positions), _exact_rotation(case, i["k"], i["w_k"], positions), i["v"].double()
        cache_k, cache_v, t = i["cache_k"].double(), i["cache_v"].double(), 0
        for s, (m, n) in enumerate(zip(news, lengths)):
            p = torch.arange(n - m, n, device="cuda")
            page = i["table"][s].long()[p // case["page"]]
            cache_k[page, :, p % case["page"]], cache_v[page, :, p % case["page"]] = k[t:t + m], v[t:t + m]
            t += m
        return {"q": q, "k": cache_k, "v": cache_v}
    out, t, group = torch.zeros(i["q"].shape, dtype=torch.float64, device="cuda"), 0, case["q_heads"] // case["kv_heads"]
    for s, (m, n) in enumerate(zip(news, lengths)):
        pages = i["table"][s, :-(-n // case["page"])].long()
        p, j = torch.arange(n - m, n, device="cuda")[:, None], torch.arange(n, device="cuda")
        hidden = torch.zeros(m, n, dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden |= j > p
        if case["window"]:
            hidden |= j <= p - case["window"]
        for h in range(case["kv_heads"]):
            k, v = (i[name][pages, h].flatten(0, 1)[:n].double() for name in ("cache_k", "cache_v"))
            for g in range(h * group, (h + 1) * group):
                a = (i["q"][t:t + m, g].double() @ k.T) / math.sqrt(case["dim"])
                out[t:t + m, g] = torch.softmax(a.masked_fill_(hidden, -math.inf), -1) @ v
        t += m
    return out
