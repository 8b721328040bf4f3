"""The stand-alone operators of a transformer block, as cases that can be timed and compared.

Four kinds, told apart by ``case["kind"]``:

  table      cosines and sines of rotary positions, scaled for contexts longer than the trained ones
  rope       rotary positions applied to heads: half-split or interleaved pairs, the whole head or its leading part
  linear     y = act(x W^T + bias) + residual
  attention  softmax attention over packed sequences of different lengths, grouped heads, causal or not, over keys that lie
             packed or in a cache with room behind each sequence

``own`` tells whether ``run`` calls the framework's kernels or computes the same from elementary torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, **kw):
    return {"name": name, **kw} if name else kw


def _table(name, positions, rotary, theta, scaling, factor, trained):
    return _case(name, kind="table", positions=positions, rotary=rotary, theta=theta, scaling=scaling, factor=factor,
                 trained=trained)


def _rope(name, dtype, tokens, heads, extra, hd, rotary, layout, transpose, max_pos):
    """`extra` heads lie behind the rotated ones in every token's row (the values of a fused projection)."""
    return _case(name, kind="rope", dtype=dtype, tokens=tokens, heads=heads, extra=extra, hd=hd, rotary=rotary,
                 layout=layout, transpose=transpose, max_pos=max_pos)


def _linear(name, dtype, m, k, n, act, bias, resid):
    return _case(name, kind="linear", dtype=dtype, m=m, k=k, n=n, act=act, bias=bias, resid=resid)


def _attention(name, dtype, heads, kv_heads, hd, batch, max_q, max_k, causal, cache):
    """The first sequence has the largest lengths, those of the others are spread from a quarter of them (see _lengths);
    max_k = 0: keys as queries (a whole prompt). `cache`: keys in a cache of max_k rows a sequence, of which the first k_len
    count."""
    return _case(name, kind="attention", dtype=dtype, heads=heads, kv_heads=kv_heads, hd=hd, batch=batch, max_q=max_q,
                 max_k=max_k, causal=causal, cache=cache)


def listed():
    return [
        # the table a server fills at start-up for a context of 128k positions, trained on 8k
        _table("table_128k_turns", 131072, 128, 5e5, "turns", 16.0, 8192),
        # one new token for each of eight sequences, far into a long context, half of the head rotated: latency
        _rope("rope_8_tokens_interleaved_part", "bf16", 8, 40, 8, 128, 64, "interleaved", False, 131072),
        # a batch of prompts: queries and keys of a fused projection's rows
        _rope("rope_16k_tokens_half", "bf16", 16384, 40, 8, 128, 128, "half", False, 8192),
        # the way back (gradient), single precision, odd sizes
        _rope("rope_f32_3993_tokens_transposed", "f32", 3993, 17, 0, 64, 64, "half", True, 4096),
        # fused projection of one token with its biases: a stream of the weights
        _linear("linear_1x4096x6144_bias", "bf16", 1, 4096, 6144, "none", True, False),
        # a few sequences' tokens through an MLP's first matrix
        _linear("linear_37x4096x12288_silu", "bf16", 37, 4096, 12288, "silu", True, False),
        # a packed batch of prompts through the output projection onto the residual stream
        _linear("linear_8192x4096x4096_resid", "bf16", 8192, 4096, 4096, "none", False, True),
        # single precision, odd sizes, everything in the epilogue
        _linear("linear_f32_601x1024x1000_gelu", "f32", 601, 1024, 1000, "gelu", True, True),
        # one token of each of 16 sequences over their caches: a stream of keys and values
        _attention("attention_decode_b16_16k", "bf16", 32, 8, 128, 16, 1, 16384, True, True),
        # prompts of different lengths, causal, grouped heads
        _attention("attention_prompts_b6_causal", "bf16", 32, 8, 128, 6, 4096, 0, True, False),
        # the active block of a bidirectional model over a long cached context, 64-wide heads of their own
        _attention("attention_block_b4_hd64", "bf16", 16, 16, 64, 4, 160, 2500, False, True),
        # single precision, causal, odd lengths, seven queries to a key head
        _attention("attention_f32_b3_causal", "f32", 14, 2, 64, 3, 333, 0, True, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["table", "rope", "rope", "linear", "linear", "linear", "attention", "attention", "attention", "attention"])
    if kind == "table":
        return _table("", _log(rng, 512, 131072), 2 * _log(rng, 16, 64), rng.choice([1e4, 5e5, 1e6]),
                      rng.choice(["none", "linear", "base", "turns", "index"]), rng.choice([2.0, 4.0, 10.0, 16.0]),
                      rng.choice([2048, 4096, 8192]))
    if kind == "rope":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        hd = rng.choice([32, 64, 128, 128, 256])
        rotary = rng.choice([hd, hd, hd // 2, max(2, hd // 2 - 6)])
        heads = rng.randint(1, 48)
        tokens = _log(rng, 1, max(1, (1 << 26) // (heads * hd * (1 if dtype == "bf16" else 2))))
        return _rope("", dtype, tokens, heads, rng.choice([0, 0, 4, 9]), hd, rotary, rng.choice(["half", "interleaved"]),
                     rng.random() < 0.25, rng.choice([2048, 8192, 131072]))
    if kind == "linear":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        size = [64 * _log(rng, 2, 192), 8 * _log(rng, 8, 1024), _log(rng, 96, 8192)]
        k, n = rng.choice(size[:2]), rng.choice(size)
        most = (8192 * 4096 * 4096) // (1 if dtype == "bf16" else 16)
        m = _log(rng, 1, max(1, min(16384, most // (k * n))))
        return _linear("", dtype, m, k, n, rng.choice(["none", "none", "relu", "gelu", "gelu_tanh", "silu"]),
                       rng.random() < 0.6, rng.random() < 0.5)
    dtype = rng.choice(["bf16", "bf16", "bf16", "bf16", "f32"])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
    group = rng.choice([1, 1, 2, 4, 7, 8])
    group = min(group, max(1, 32 // kv_heads))
    hd = rng.choice([64, 128, 128]) if dtype == "bf16" else rng.choice([32, 64, 128, 256])
    batch = rng.randint(1, 16)
    heads = kv_heads * group
    form = rng.choice(["token", "block", "prompt"])
    most = (6 * 32 * 4096 * 4096) // (1 if dtype == "bf16" else 64)         # score entries of the largest listed cases
    if form == "token":
        max_k = _log(rng, 1, min(65536, (16 * 16384 * 8 * 128) // (batch * kv_heads * hd * (1 if dtype == "bf16" else 8))))
        return _attention("", dtype, heads, kv_heads, hd, batch, 1, max_k, True, True)
    if form == "block":
        max_q = rng.randint(2, 160)
        max_k = _log(rng, max_q, max(max_q + 1, min(16384, most // (batch * heads * 160))))
        return _attention("", dtype, heads, kv_heads, hd, batch, max_q, max_k, rng.random() < 0.5, True)
    max_q = _log(rng, 1, int(min(8192, math.sqrt(most // (batch * heads)))))
    return _attention("", dtype, heads, kv_heads, hd, batch, max_q, 0, rng.random() < 0.7, False)


# ---------------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, std, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _lengths(case):
    """Query and key lengths of the case's sequences: the largest, then spread over (1/4, 1) of it in an irregular order."""
    def spread(most, step):
        return [most] + [math.ceil(most * (0.25 + 0.75 * (b * step % 1.0))) for b in range(1, case["batch"])]
    q = spread(case["max_q"], 0.6180339887498949)
    return q, q if case["max_k"] == 0 else [max(a, b) for a, b in zip(q, spread(case["max_k"], 0.7548776662466927))]


def _frequencies(rotary, theta, scaling, factor, trained, low=1.0, high=32.0):
    """Angle a position of each pair, float64 [rotary / 2]."""
    j = torch.arange(rotary // 2, dtype=torch.float64, device="cuda")
    if scaling == "base" and rotary > 2:
        theta = theta * factor ** (rotary / (rotary - 2))
    f = theta ** (-2.0 * j / rotary)
    if scaling == "linear":
        f = f / factor
    elif scaling == "turns":
        keep = ((trained * f / (2.0 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        f = keep * f + (1.0 - keep) * f / factor
    elif scaling == "index":
        at = lambda turns: rotary * math.log(trained / (2.0 * math.pi * turns)) / (2.0 * math.log(theta))
        first, last = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rotary - 1)
        keep = 1.0 - ((j - first) / max(last - first, 1e-3)).clamp(0.0, 1.0)
        f = keep * f + (1.0 - keep) * f / factor
    return f


def prepare(case, seed):
    g, kind = _generator(seed), case["kind"]
    if kind == "table":
        # (the magnitude goes with the seed: another seed, another table)
        return {"case": case, "magnitude": 1.0 + (seed % 1009) / 1009.0}
    dt = DT[case["dtype"]]
    if kind == "rope":
        row = case["heads"] + case["extra"]
        x = _normal(g, (case["tokens"], row, case["hd"]), 1.0, dt)[:, :case["heads"]]
        angle = torch.arange(case["max_pos"], dtype=torch.float64, device="cuda")[:, None] * \
            _frequencies(case["rotary"], 5e5, "none", 1.0, 0)
        table = torch.stack((angle.cos(), angle.sin()), -1).float()
        pos = torch.randint(0, case["max_pos"], (case["tokens"],), generator=g, device="cuda", dtype=torch.int32)
        return {"case": case, "x": x, "table": table, "positions": pos}
    if kind == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"case": case, "x": _normal(g, (m, k), 1.0, dt), "w": _normal(g, (n, k), k ** -0.5, dt),
                "bias": _normal(g, (n,), 0.5, torch.float32) if case["bias"] else None,
                "resid": _normal(g, (m, n), 1.0, dt) if case["resid"] else None}
    batch, hd = case["batch"], case["hd"]
    q_len, k_len = _lengths(case)
    if case["cache"]:
        room = max(max(k_len), 1)
        k_begin, rows = [b * room for b in range(batch)], batch * room
    else:
        k_begin, rows = [sum(k_len[:b]) for b in range(batch)], sum(k_len)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    q_begin = [sum(q_len[:b]) for b in range(batch + 1)]
    return {"case": case, "q": _normal(g, (q_begin[-1], case["heads"], hd), 1.0, dt),
            "k": _normal(g, (rows, case["kv_heads"], hd), 1.0, dt), "v": _normal(g, (rows, case["kv_heads"], hd), 1.0, dt),
            "q_begin": ints(q_begin), "k_begin": ints(k_begin), "k_len": ints(k_len), "most_q": max(q_len), "most_k": max(k_len)}


# ---------------------------------------------------------------------------------------------------------------
def _plain_rope(s):
    case, x, r = s["case"], s["x"], s["case"]["rotary"]
    cs = s["table"][s["positions"].long()][:, None]                    # [tokens, 1, r / 2, 2]
    cos, sin = cs[..., 0], cs[..., 1]
    if case["transpose"]:
        sin = -sin
    y = x.float()
    if case["layout"] == "half":
        a, b = y[..., :r // 2], y[..., r // 2:r]
        rot = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = y[..., :r:2], y[..., 1:r:2]
        rot = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((rot, y[..., r:]), -1).to(x.dtype)


def _act(y, name):
    if name == "relu":
        return y.clamp(min=0.0)
    if name == "silu":
        return y / (1.0 + torch.exp(-y))
    if name == "gelu":
        return 0.5 * y * (1.0 + torch.erf(y * 0.5 ** 0.5))
    if name == "gelu_tanh":
        return 0.5 * y * (1.0 + torch.tanh((2.0 / math.pi) ** 0.5 * (y + 0.044715 * y ** 3)))
    return y


def _plain_linear(s):
    y = s["x"].float() @ s["w"].float().T
    if s["bias"] is not None:
        y = y + s["bias"]
    y = _act(y, s["case"]["act"])
    if s["resid"] is not None:
        y = y + s["resid"].float()
    return y.to(s["x"].dtype)


def _plain_attention(s):
    case = s["case"]
    batch, hd, kvh = case["batch"], case["hd"], case["kv_heads"]
    grp, nq, nk = case["heads"] // kvh, s["most_q"], s["most_k"]
    begin, q_len, k_len = s["q_begin"][:-1].long(), s["q_begin"].diff(), s["k_len"]
    iq, ik = torch.arange(nq, device="cuda"), torch.arange(nk, device="cuda")
    # sequences side by side: [batch, kv head, group * query, hd] and [batch, kv head, key, hd]
    rows_q = (begin[:, None] + iq).clamp(max=s["q"].shape[0] - 1)
    rows_k = (s["k_begin"].long()[:, None] + ik).clamp(max=s["k"].shape[0] - 1)
    q = s["q"][rows_q].float().view(batch, nq, kvh, grp, hd).permute(0, 2, 3, 1, 4).reshape(batch, kvh, grp * nq, hd)
    k, v = s["k"][rows_k].float().transpose(1, 2), s["v"][rows_k].float().transpose(1, 2)
    scores = (q @ k.transpose(-1, -2)).mul_(hd ** -0.5).view(batch, kvh, grp, nq, nk)
    hidden = (ik >= k_len[:, None])[:, None, None, None, :]
    if case["causal"]:
        hidden = hidden | (ik > (iq[:, None] + (k_len - q_len)[:, None, None]))[:, None, None]
    scores = scores.masked_fill_(hidden, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(batch, kvh, grp * nq, nk) @ v).view(batch, kvh, grp, nq, hd) / total
    lse = (top + total.log()).squeeze(-1)
    there = iq < q_len[:, None]                                       # [batch, query]
    o = o.permute(0, 3, 1, 2, 4).reshape(batch, nq, kvh * grp, hd)[there]
    lse = lse.permute(0, 3, 1, 2).reshape(batch, nq, kvh * grp)[there]
    return o.to(s["q"].dtype), lse


def run(state):
    case = state["case"]
    kind = case["kind"]
    if own:
        from paper_2605_08134_b200 import dare
        if kind == "table":
            return dare.rope_table(case["positions"], case["rotary"], case["theta"], scaling=dare.ROPE_SCALE[case["scaling"]],
                                   factor=case["factor"], trained=case["trained"], low=1.0, high=32.0,
                                   magnitude=state["magnitude"], device="cuda")
        if kind == "rope":
            return dare.rope(state["x"], state["table"], state["positions"], layout=dare.ROPE_LAYOUT[case["layout"]],
                             transpose=case["transpose"])
        if kind == "linear":
            return dare.linear(state["x"], state["w"], bias=state["bias"], act=dare.ACT[case["act"]], resid=state["resid"])
        return dare.attention(state["q"], state["k"], state["v"], state["q_begin"], state["k_begin"], k_len=state["k_len"],
                              causal=case["causal"], return_lse=True)
    if kind == "table":
        angle = torch.arange(case["positions"], dtype=torch.float64, device="cuda")[:, None] * \
            _frequencies(case["rotary"], case["theta"], case["scaling"], case["factor"], case["trained"])
        return torch.stack((angle.cos() * state["magnitude"], angle.sin() * state["magnitude"]), -1).float()
    if kind == "rope":
        return _plain_rope(state)
    if kind == "linear":
        return _plain_linear(state)
    return _plain_attention(state)


# ---------------------------------------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "table":
        n = case["positions"] * case["rotary"]
        return {"bytes": 4 * n, "flops": n}
    e = 2 if case["dtype"] == "bf16" else 4
    if kind == "rope":
        n = case["tokens"] * case["heads"] * case["hd"]
        rows = min(case["tokens"], case["max_pos"])
        return {"bytes": 2 * n * e + 4 * case["tokens"] + 4 * rows * case["rotary"],
                "flops": 3 * case["tokens"] * case["heads"] * case["rotary"]}
    if kind == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": e * (m * k + n * k + m * n * (2 if case["resid"] else 1)) + (4 * n if case["bias"] else 0),
                "flops": 2 * m * n * k}
    q, k = _lengths(case)
    pairs = sum(a * b - (a * (a - 1) // 2 if case["causal"] else 0) for a, b in zip(q, k))
    hd = case["hd"]
    return {"bytes": int(e * hd * (2 * sum(q) * case["heads"] + 2 * sum(k) * case["kv_heads"]) + 4 * sum(q) * case["heads"]),
            "flops": int(4 * hd * case["heads"] * pairs)}


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "table":
        # complex exponentials of the turn's remainder
        f = _frequencies(case["rotary"], case["theta"], case["scaling"], case["factor"], case["trained"])
        a = torch.outer(torch.arange(case["positions"], dtype=torch.float64, device="cuda"), f)
        return torch.view_as_real(torch.polar(torch.full_like(a, s["magnitude"]), a))
    if kind == "rope":
        r, x = case["rotary"], s["x"].double()
        turn = torch.view_as_complex(s["table"].double())[s["positions"].long()]
        if case["transpose"]:
            turn = turn.conj()
        part = x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2) if case["layout"] == "half" else x[..., :r].unflatten(-1, (r // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(part.contiguous()) * turn[:, None, :])
        z = z.transpose(-1, -2) if case["layout"] == "half" else z
        return torch.cat((z.flatten(-2), x[..., r:]), -1)
    if kind == "linear":
        y = torch.einsum("mk,nk->mn", s["x"].double(), s["w"].double())
        if s["bias"] is not None:
            y += s["bias"].double()
        act = {"none": lambda t: t, "relu": torch.relu, "silu": lambda t: t * torch.sigmoid(t),
               "gelu": lambda t: t * torch.special.ndtr(t),
               "gelu_tanh": lambda t: t * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (t + 0.044715 * t * t * t))}[case["act"]]
        y = act(y)
        return y if s["resid"] is None else y + s["resid"].double()
    if case["batch"] * case["heads"] * s["most_q"] * s["most_k"] > 8 << 30:
        return None, None
    q_at, k_at, k_len = s["q_begin"].tolist(), s["k_begin"].tolist(), s["k_len"].tolist()
    grp, outs, sums = case["heads"] // case["kv_heads"], [], []
    for b in range(case["batch"]):
        n, m = q_at[b + 1] - q_at[b], k_len[b]
        q = s["q"][q_at[b]:q_at[b + 1]].double()
        per_head = []
        for h in range(case["heads"]):
            k, v = (s[c][k_at[b]:k_at[b] + m, h // grp].double() for c in "kv")
            z = q[:, h] @ k.T / math.sqrt(case["hd"])
            if case["causal"]:
                z += torch.full((n, m), -math.inf, dtype=torch.float64, device="cuda").triu(m - n + 1)
            lse = torch.logsumexp(z, 1)
            per_head.append(((z - lse[:, None]).exp() @ v, lse))
        outs.append(torch.stack([o for o, _ in per_head], 1))
        sums.append(torch.stack([e for _, e in per_head], 1))
    return torch.cat(outs), torch.cat(sums)
