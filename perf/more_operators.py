"""Cases of a decode step that holds its cache, and some of its weights, in 4 bits, and ends in a token.

A case is a dict of plain values; `op` names the entry points:

  cache      cache_write4 and cache_read4: new tokens' keys and values rounded into 4-bit caches, and the caches given
             back in 16 bits
  attention  prefix_attention4: the new tokens of a batch over a shared prefix and the sequences' own caches, both in
             4 bits; with `weights`, also the weight that each own key has gathered
  gemv       gemv4: products with a matrix of 4-bit codes that groups of columns share scales (and bases) of
  sample     sample: a token of each row of logits by temperature, top-k, top-p and min-p, from given random numbers

A 4-bit row of `dim` columns (a multiple of 32) is dim/2 bytes of codes, dim/32 pairs (scale, base) of bfloat16 and zeros
up to a multiple of 16 bytes. Byte n*(dim/32)+g has the codes of columns 32g+2n (its low half) and 32g+2n+1, and every 32
neighbouring columns share a pair: value = base + scale * (code - 8).

Head counts, head sizes and widths are those of the 7B, 8B and 70B shapes of this repository's workloads (32 or 64 heads
of 128 on 8 or 32 of keys; 4096 and 8192 wide; batches of 1 to 16), and generic ones; the numbers of logits are generic.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
LEAST = 2.0**-40  # of the greatest weight: lighter tokens are never drawn


def listed():
    return [
        # a decode step's new tokens into short caches
        {"name": "cache b16 t1", "op": "cache", "type": "bf16", "batch": 16, "tokens": 1, "kv_heads": 8, "dim": 128,
         "own": 64},
        # a long prompt's keys and values, and back
        {"name": "cache b1 t16384", "op": "cache", "type": "bf16", "batch": 1, "tokens": 16384, "kv_heads": 8,
         "dim": 128, "own": 16384},
        # one chat at its start, 8B shape: a short system prompt and a few hundred tokens
        {"name": "attn b1 p512", "op": "attention", "type": "bf16", "batch": 1, "queries": 1, "heads": 32,
         "kv_heads": 8, "dim": 128, "prefix": 512, "own": 300, "weights": False},
        # speculative decoding of three tokens, 7B shape (a key head for each head), odd lengths
        {"name": "attn b5 q3 p1777 f16", "op": "attention", "type": "f16", "batch": 5, "queries": 3, "heads": 32,
         "kv_heads": 32, "dim": 128, "prefix": 1777, "own": 777, "weights": False},
        # a decode batch of the 70B shape with long caches of its own, that gathers the weights an eviction goes by
        {"name": "attn b16 own16384 weights", "op": "attention", "type": "bf16", "batch": 16, "queries": 1,
         "heads": 64, "kv_heads": 8, "dim": 128, "prefix": 2048, "own": 16384, "weights": True},
        # the sequences' own prompts, a chunk of 256 tokens each, on the shared one
        {"name": "attn b4 q256 p4096", "op": "attention", "type": "bf16", "batch": 4, "queries": 256, "heads": 32,
         "kv_heads": 8, "dim": 128, "prefix": 4096, "own": 512, "weights": False},
        # a square projection in a decode step of one sequence
        {"name": "gemv 4096x4096 b1", "op": "gemv", "type": "bf16", "batch": 1, "rows": 4096, "cols": 4096,
         "group": 128, "scale": "bf16", "bases": False},
        # a small odd matrix with fine groups, for a few sequences
        {"name": "gemv 1021x4128 b5 f16", "op": "gemv", "type": "f16", "batch": 5, "rows": 1021, "cols": 4128,
         "group": 32, "scale": "f16", "bases": True},
        # the gate projection of the 70B shape for a full decode batch
        {"name": "gemv 28672x8192 b16", "op": "gemv", "type": "bf16", "batch": 16, "rows": 28672, "cols": 8192,
         "group": 64, "scale": "bf16", "bases": True},
        # the end of one chat's step
        {"name": "sample 1x32000", "op": "sample", "type": "f32", "rows": 1, "vocab": 32000, "temperature": 0.8,
         "top_k": 50, "top_p": 0.95, "min_p": 0.0, "mixed": False, "masked": False},
        # requests with settings of their own in one batch, some tokens ruled out, logits of which many are equal
        {"name": "sample 61x50001 mixed", "op": "sample", "type": "bf16", "rows": 61, "vocab": 50001,
         "temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0, "mixed": True, "masked": True},
        # a large batch of continuations drawn from most of the tokens
        {"name": "sample 256x131072", "op": "sample", "type": "f32", "rows": 256, "vocab": 131072, "temperature": 1.0,
         "top_k": 0, "top_p": 0.9, "min_p": 0.0, "mixed": False, "masked": False},
    ]


# What a drawn case may cost at most: the largest listed ones.
MOST_BYTES = {"cache": 16384 * 8 * 2 * (256 + 80), "attention": 188 << 20, "gemv": 128 << 20}
MOST_SCORES = 160 << 20  # scores of a plain pass
MOST_LOGITS = 256 * 131072


def _log(rng, low, high):
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def _draw_cache(rng):
    case = {"op": "cache", "type": rng.choice(["bf16", "f16"]), "batch": rng.randint(1, 16),
            "tokens": rng.choice([1, rng.randint(2, 8), _log(rng, 9, 16384)]), "kv_heads": rng.choice([1, 4, 8, 32]),
            "dim": rng.choice([64, 96, 128, 128, 256])}
    case["own"] = max(case["tokens"], _log(rng, 1, 16384))
    while work(case)["bytes"] > MOST_BYTES["cache"]:
        case["tokens"], case["own"] = case["tokens"] // 2 + 1, case["own"] // 2 + 1
        case["own"] = max(case["own"], case["tokens"])
    return case


def _draw_attention(rng):
    heads, kv_heads = rng.choice([(32, 8), (64, 8), (32, 32), (16, 2), (24, 8)])
    case = {"op": "attention", "type": rng.choice(["bf16", "f16"]), "batch": rng.randint(1, 16),
            "queries": rng.choice([1, 1, 1, rng.randint(2, 8), _log(rng, 9, 256)]), "heads": heads,
            "kv_heads": kv_heads, "dim": rng.choice([64, 96, 128, 128]), "prefix": _log(rng, 1, 131072),
            "own": 0, "weights": False}
    case["own"] = max(case["queries"], _log(rng, 1, 16384))
    case["weights"] = case["queries"] <= 8 and rng.random() < 0.4
    rows = case["batch"] * case["queries"] * heads
    while rows * (case["prefix"] + case["own"]) > MOST_SCORES or work(case)["bytes"] > MOST_BYTES["attention"]:
        if case["prefix"] >= case["own"] or case["own"] == case["queries"]:
            case["prefix"] = case["prefix"] // 2 + 1
        else:
            case["own"] = max(case["queries"], case["own"] // 2)
    return case


def _draw_gemv(rng):
    group = rng.choice([32, 64, 128])
    case = {"op": "gemv", "type": rng.choice(["bf16", "f16"]), "batch": rng.choice([1, 1, rng.randint(2, 16)]),
            "rows": _log(rng, 256, 32768), "cols": _log(rng, 256, 32768) // group * group, "group": group,
            "scale": rng.choice(["bf16", "f16"]), "bases": rng.random() < 0.5}
    # heights are multiples of 16; now and then they are any number
    step = rng.choice([16, 16, 1])
    case["rows"] = case["rows"] // step * step
    while work(case)["bytes"] > MOST_BYTES["gemv"]:
        case["rows"] = case["rows"] // 2 // step * step
    return case


def _draw_sample(rng):
    vocab = _log(rng, 500, 200000)
    case = {"op": "sample", "type": rng.choice(["f32", "bf16", "f16"]), "rows": 0, "vocab": vocab,
            "temperature": rng.choice([0.0, 0.6, 0.8, 1.0, 1.3]), "top_k": rng.choice([0, 0, 20, 50, _log(rng, 1, vocab)]),
            "top_p": rng.choice([1.0, 0.9, 0.95, rng.uniform(0.05, 0.99)]), "min_p": rng.choice([0.0, 0.0, 0.05, 0.2]),
            "mixed": rng.random() < 0.4, "masked": rng.random() < 0.3}
    case["rows"] = _log(rng, 1, min(512, MOST_LOGITS // vocab))
    return case


def draw(rng):
    return rng.choice([_draw_cache, _draw_attention, _draw_attention, _draw_gemv, _draw_sample])(rng)


def _row_bytes(dim):
    return (dim // 2 + dim // 8 + 15) // 16 * 16


def _lens(case):
    """Lengths of the sequences' own caches, the new tokens with them, spread between the least and the capacity."""
    low, high, b = case["queries"] if case["op"] == "attention" else case["tokens"], case["own"], case["batch"]
    return [high - (high - low) * i // b if i else high for i in range(b)]


def work(case):
    if case["op"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * BYTES[case["type"]] + 12 * case["rows"], "flops": 4 * n}
    if case["op"] == "gemv":
        n, b = case["rows"] * case["cols"], case["batch"]
        scales = n // case["group"] * 2 * (2 if case["bases"] else 1)
        return {"bytes": n // 2 + scales + 2 * b * case["cols"] + 4 * b * case["rows"], "flops": 2 * b * n}
    d, h, b = case["dim"], case["kv_heads"], case["batch"]
    row = d // 2 + d // 8
    if case["op"] == "cache":
        new, held = 2 * b * case["tokens"] * h, 2 * b * case["own"] * h
        return {"bytes": new * (2 * d + row) + held * (row + 2 * d), "flops": 8 * new * d + 2 * held * d}
    n, q = sum(_lens(case)), case["queries"]
    seen = q * (b * case["prefix"] + n) - b * q * (q - 1) // 2
    more = 8 * b * h * case["own"] if case["weights"] else 0
    return {"bytes": 2 * row * h * (case["prefix"] + n) + 4 * b * q * case["heads"] * d + more,
            "flops": 4 * d * case["heads"] * seen}


def _rand(g, shape, scale=1.0, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def _keys(g, shape, dtype):
    """Keys or values [.., heads, dim]: tokens differ, and each head has channels that stand out in all of them."""
    t = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    t += _rand(g, shape[-2:], 0.5)
    return t.to(dtype)


def _cache(g, shape, dim):
    """4-bit rows of tokens [.., heads] as a cache holds them: codes in the middle more often, and 32 columns' scale
    and base."""
    t = torch.zeros((*shape, _row_bytes(dim)), dtype=torch.uint8, device="cuda")
    half = dim // 2
    low, high = (torch.randn((*shape, half), generator=g, device="cuda", dtype=torch.float16).mul_(3.2).add_(8)
                 .round_().clamp_(0, 15).to(torch.uint8) for _ in range(2))
    t[..., :half] = low | high << 4
    pairs = torch.empty((*shape, dim // 32, 2), dtype=torch.bfloat16, device="cuda")
    pairs[..., 0] = 0.28 + 0.08 * torch.rand((*shape, dim // 32), generator=g, device="cuda")
    pairs[..., 1] = _rand(g, (*shape, dim // 32), 0.3) + _rand(g, (shape[-1], dim // 32), 0.3)
    t[..., half:half + dim // 8] = pairs.flatten(-2).view(torch.uint8)
    return t


def _logits(case, g):
    rows, n = case["rows"], case["vocab"]
    x = torch.randn((rows, n), generator=g, device="cuda").mul_(2.2)
    few = min(n, 40)  # what the text so far makes likely
    each = n // few
    at = each * torch.arange(few, device="cuda") + torch.randint(0, each, (rows, few), generator=g, device="cuda")
    x.scatter_(1, at, 4 + 3 * torch.rand((rows, few), generator=g, device="cuda")
               + 6 * torch.rand((rows, 1), generator=g, device="cuda"))
    x = x.to(TYPE[case["type"]])
    if case["masked"]:  # a grammar's: all but some of the tokens ruled out, in some rows
        out = torch.rand((rows, n), generator=g, device="cuda") < torch.rand((rows, 1), generator=g, device="cuda") ** 0.1
        out &= torch.rand((rows, 1), generator=g, device="cuda") < 0.5
        out[:, n // 2] = False
        x.masked_fill_(out, -math.inf)
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    state = {"case": dict(case)}
    if case["op"] == "sample":
        rows = case["rows"]
        state["logits"] = _logits(case, g)
        state["uniforms"] = torch.rand((rows,), generator=g, device="cuda")
        for name in ("temperature", "top_k", "top_p", "min_p"):
            state[name] = case[name]
        if case["mixed"]:
            pick = lambda values: torch.tensor(values, device="cuda")[  # noqa: E731
                torch.randint(0, len(values), (rows,), generator=g, device="cuda")]
            state["temperature"] = pick([0.0, 0.5, 0.7, 1.0, 1.0, 1.5])
            state["top_k"] = pick([0, 1, 20, 50, 1000]).int()
            state["top_p"] = pick([1.0, 0.95, 0.9, 0.5])
            state["min_p"] = pick([0.0, 0.0, 0.05, 0.1])
        return state
    if case["op"] == "gemv":
        rows, cols, scale = case["rows"], case["cols"], TYPE[case["scale"]]
        state["codes"] = torch.randint(0, 256, (rows, cols // 2), generator=g, device="cuda", dtype=torch.uint8)
        shape = (rows, cols // case["group"])
        state["scales"] = (0.002 + 0.004 * torch.rand(shape, generator=g, device="cuda")).to(scale)
        state["bases"] = _rand(g, shape, 0.004, scale) if case["bases"] else None
        # activations: a few channels far larger than the rest
        size = 1 + 20 * (torch.rand(cols, generator=g, device="cuda") < 0.005).float()
        state["x"] = (_rand(g, (case["batch"], cols)) * size).to(TYPE[case["type"]])
        return state
    b, h, d, dtype = case["batch"], case["kv_heads"], case["dim"], TYPE[case["type"]]
    order = torch.randperm(b, generator=g, device="cuda")
    state["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")[order].contiguous()
    state["cache_k"], state["cache_v"] = (_cache(g, (b, case["own"], h), d) for _ in range(2))
    if case["op"] == "cache":
        state["k"], state["v"] = (_keys(g, (b, case["tokens"], h, d), dtype) for _ in range(2))
        return state
    state["q"] = _rand(g, (b, case["queries"], case["heads"], d), 2.0, dtype)
    state["prefix_k"], state["prefix_v"] = (_cache(g, (case["prefix"], h), d) for _ in range(2))
    if case["weights"]:
        # gathered weight falls off steeply: a few tokens hold most, many have next to none
        u = torch.rand((b, h, case["own"]), generator=g, device="cuda").clamp_(min=1e-3)
        state["weights"] = u.pow_(-1.2).mul_(1e-3)
    return state


def _values(rows, dim):
    """Values [.., dim] in float32 that 4-bit rows stand for."""
    half, groups = dim // 2, dim // 32
    b = rows[..., :half].unflatten(-1, (16, groups)).transpose(-1, -2)            # .., group, pair of columns
    codes = torch.stack([b & 15, b >> 4], -1).flatten(-2).float()                 # .., group, 32
    pairs = rows[..., half:half + dim // 8].contiguous().view(torch.bfloat16).float().unflatten(-1, (groups, 2))
    return (pairs[..., 1:] + pairs[..., :1] * (codes - 8)).flatten(-2)


def _rows(x):
    """The 4-bit rows of x [.., dim]."""
    dim = x.shape[-1]
    groups = dim // 32
    t = x.float().unflatten(-1, (groups, 32))
    low, high = t.amin(-1, keepdim=True), t.amax(-1, keepdim=True)
    over = lambda n: torch.full_like(low, n)  # noqa: E731  (a number as a divisor may be multiplied with its reciprocal)
    base = ((7 * low + 8 * high) / over(15)).bfloat16().float()
    scale = torch.maximum((high - base) / over(7), (base - low) / over(8)).bfloat16().float()
    good = base.isfinite() & scale.isfinite() & t.isfinite().all(-1, keepdim=True)
    # which whole number is nearest needs more bits than 32
    codes = ((t.double() - base.double()) / scale.double()).round().clamp(-8, 7) + 8
    codes = torch.where(good & (scale > 0), codes, torch.full_like(codes, 8.0)).to(torch.uint8)
    pairs = torch.where(good, torch.cat([scale, base], -1), torch.full_like(scale, math.nan)).bfloat16()
    codes = codes.unflatten(-1, (16, 2))                                          # .., group, pair of columns, 2
    b = (codes[..., 0] | codes[..., 1] << 4).transpose(-1, -2).flatten(-2)
    out = torch.zeros((*x.shape[:-1], _row_bytes(dim)), dtype=torch.uint8, device=x.device)
    out[..., :dim // 2] = b
    out[..., dim // 2:dim // 2 + dim // 8] = pairs.flatten(-2).view(torch.uint8)
    return out


def _plain_cache(s):
    b, n = s["k"].shape[:2]
    slots = s["lens"].long()[:, None] - n + torch.arange(n, device=s["k"].device)
    at = torch.arange(b, device=s["k"].device)[:, None]
    outs = {}
    for name in ("k", "v"):
        cache = s["cache_" + name]
        cache[at, slots] = _rows(s[name])
        outs[name] = _values(cache, s["case"]["dim"]).to(s[name].dtype)
    return outs


def _plain_attention(s):
    d = s["case"]["dim"]
    q, k, v, pk, pv = s["q"].float(), *(_values(s[n], d) for n in ("cache_k", "cache_v", "prefix_k", "prefix_v"))
    b, n_q, heads, _ = q.shape
    h, g, cap, p = k.shape[2], heads // k.shape[2], k.shape[1], pk.shape[0]
    rows = q.view(b, n_q, h, g, d).permute(2, 0, 1, 3, 4).contiguous()            # h, b, q, g, d
    scale = 1 / math.sqrt(d)
    on_prefix = torch.matmul(rows.view(h, b * n_q * g, d), pk.permute(1, 2, 0).contiguous()) * scale
    mine = rows.view(h, b, n_q * g, d).transpose(0, 1).contiguous()               # b, h, q*g, d
    on_own = torch.matmul(mine, k.permute(0, 2, 3, 1).contiguous()) * scale       # b, h, q*g, cap
    at = torch.arange(cap, device=q.device)
    back = torch.arange(n_q - 1, -1, -1, device=q.device)
    seen = at[None, None, :] < s["lens"].long()[:, None, None] - back[None, :, None]  # b, q, cap
    seen = seen[:, None, :, None, :].expand(b, h, n_q, g, cap).reshape(b, h, n_q * g, cap)
    on_own = on_own.masked_fill(~seen, -math.inf)
    on_prefix = on_prefix.view(h, b, n_q * g, p).transpose(0, 1)                  # b, h, q*g, p
    most = torch.maximum(on_prefix.amax(-1, keepdim=True), on_own.amax(-1, keepdim=True))
    e_prefix, e_own = torch.exp(on_prefix - most), torch.exp(on_own - most)
    total = e_prefix.sum(-1, keepdim=True) + e_own.sum(-1, keepdim=True)
    flat = e_prefix.transpose(0, 1).reshape(h, b * n_q * g, p)
    o = torch.matmul(flat, pv.transpose(0, 1).contiguous()).view(h, b, n_q * g, d).transpose(0, 1)
    o = (o + torch.matmul(e_own, v.transpose(1, 2).contiguous())) / total
    outs = {"out": o.reshape(b, h, n_q, g, d).permute(0, 2, 1, 3, 4).reshape(b, n_q, heads, d).to(s["q"].dtype)}
    if s["case"]["weights"]:
        outs["weights"] = s["weights"] + (e_own / total).sum(2)
    return outs


def _plain_gemv(s):
    rows, groups = s["scales"].shape
    codes = torch.stack([s["codes"] & 15, s["codes"] >> 4], -1).view(rows, groups, -1).float()
    w = s["scales"].float()[..., None] * (codes - 8)
    if s["bases"] is not None:
        w = w + s["bases"].float()[..., None]
    return torch.matmul(s["x"].float(), w.view(rows, -1).t())


def _plain_sample(s):
    x = s["logits"].double()
    x = torch.where(x.isnan(), torch.full_like(x, -math.inf), x)
    rows, n = x.shape
    column = lambda v: (v if torch.is_tensor(v) else torch.full((rows,), v, device=x.device))[:, None]  # noqa: E731
    temperature, top_p, min_p = (column(s[name]).float().double() for name in ("temperature", "top_p", "min_p"))
    top_k = column(s["top_k"]).long()
    greedy = temperature <= 0
    most = x.amax(1, keepdim=True)
    w = torch.exp((x - most) / torch.where(greedy, torch.ones_like(temperature), temperature))
    w = torch.where(x == most, torch.ones_like(w), torch.where(w < LEAST, torch.zeros_like(w), w))
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    w = torch.gather(w, 1, order)
    k = torch.where((top_k <= 0) | (top_k > n), torch.full_like(top_k, n), top_k)
    k = torch.where(greedy, torch.ones_like(k), k)
    at = torch.arange(n, device=x.device)
    w = torch.where(at < k, w, torch.zeros_like(w))
    before = torch.cumsum(w, 1)
    enough = (before < top_p * before[:, -1:]) & (top_p < 1)
    w = torch.where((at == 0) | (top_p >= 1) | torch.roll(enough, 1, 1), w, torch.zeros_like(w))
    w = torch.where((w >= min_p) | (at == 0), w, torch.zeros_like(w))
    w = torch.zeros_like(w).scatter_(1, order, w)                                 # by index again
    before = torch.cumsum(w, 1)
    total = before[:, -1:]
    past = (before > s["uniforms"].double()[:, None] * total) & (w > 0)
    token = torch.where(past.any(1), past.int().argmax(1), n - 1 - (w > 0).flip(1).int().argmax(1))
    logprob = torch.log(torch.gather(w, 1, token[:, None]) / total)[:, 0]
    return {"tokens": token.int(), "logprobs": logprob.float()}


def _own_cache(s):
    import paper_2502_00922_amd as hl
    hl.cache_write4(s["k"], s["v"], s["cache_k"], s["cache_v"], s["lens"])
    d, dtype = s["case"]["dim"], s["k"].dtype
    return {"k": hl.cache_read4(s["cache_k"], d, dtype), "v": hl.cache_read4(s["cache_v"], d, dtype)}


def _own_attention(s):
    import paper_2502_00922_amd as hl
    r = hl.prefix_attention4(s["q"], s["cache_k"], s["cache_v"], s["lens"], prefix_k=s["prefix_k"],
                             prefix_v=s["prefix_v"], weights=s["weights"] if s["case"]["weights"] else None)
    return {"out": r[0], "weights": r[1]} if s["case"]["weights"] else {"out": r[0]}


def _own_gemv(s):
    import paper_2502_00922_amd as hl
    return hl.gemv4(s["codes"], s["scales"], s["x"], bases=s["bases"])


def _own_sample(s):
    import paper_2502_00922_amd as hl
    r = hl.sample(s["logits"], s["uniforms"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                  min_p=s["min_p"])
    return {"tokens": r.tokens, "logprobs": r.logprobs}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"cache": _own_cache, "attention": _own_attention, "gemv": _own_gemv, "sample": _own_sample}[op](state)
    return {"cache": _plain_cache, "attention": _plain_attention, "gemv": _plain_gemv, "sample": _plain_sample}[op](state)


def _numbers(rows, dim):
    """What 4-bit rows stand for, in 64 bits, a group at a time."""
    groups, out = dim // 32, torch.empty((*rows.shape[:-1], dim), dtype=torch.float64, device=rows.device)
    pairs = rows[..., dim // 2:dim // 2 + dim // 8].contiguous().view(torch.bfloat16).double()
    for g in range(groups):
        scale, base = pairs[..., 2 * g:2 * g + 1], pairs[..., 2 * g + 1:2 * g + 2]
        b = rows[..., g:dim // 2:groups]
        out[..., 32 * g:32 * g + 32:2] = base + scale * (b.remainder(16).double() - 8)
        out[..., 32 * g + 1:32 * g + 32:2] = base + scale * (b.div(16, rounding_mode="floor").double() - 8)
    return out


def _rounded(x):
    """x (float32) to bfloat16, ties to even."""
    bits = x.view(np.uint32).astype(np.uint64)
    return ((bits + 0x7FFF + (bits >> 16 & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)


def _exact_cache(case, s):
    lens, d, n = s["lens"].tolist(), case["dim"], case["tokens"]
    outs = {}
    for name in ("k", "v"):
        held = _numbers(s["cache_" + name], d)
        x = s[name].float().cpu().numpy().reshape(case["batch"], n, case["kv_heads"], d // 32, 32)
        low, high = x.min(-1), x.max(-1)
        base = _rounded((np.float32(7) * low + np.float32(8) * high) / np.float32(15))
        scale = _rounded(np.maximum((high - base) / np.float32(7), (base - low) / np.float32(8)))
        x, base, scale = (t.astype(np.float64) for t in (x, base[..., None], scale[..., None]))
        steps = np.clip(np.rint((x - base) / np.where(scale > 0, scale, 1)), -8, 7)
        new = torch.from_numpy((base + scale * steps).reshape(case["batch"], n, case["kv_heads"], d)).to("cuda")
        for b in range(case["batch"]):
            held[b, lens[b] - n:lens[b]] = new[b]
        outs[name] = held
    return outs


def _exact_attention(case, s):
    b, n_q, heads, d = s["q"].shape
    g = heads // case["kv_heads"]
    out = torch.zeros((b, n_q, heads, d), dtype=torch.float64, device="cuda")
    gathered = s["weights"].double() if case["weights"] else None
    lens = s["lens"].tolist()
    for head in range(case["kv_heads"]):
        shared_k, shared_v = (_numbers(s[name][:, head], d) for name in ("prefix_k", "prefix_v"))
        for i in range(b):
            keys = torch.cat([shared_k, _numbers(s["cache_k"][i, :lens[i], head], d)])
            values = torch.cat([shared_v, _numbers(s["cache_v"][i, :lens[i], head], d)])
            rows = s["q"][i, :, head * g:(head + 1) * g].double().reshape(n_q * g, d)
            scores = rows @ keys.t().contiguous() / math.sqrt(d)
            last = case["prefix"] + lens[i] - n_q + torch.arange(n_q, device="cuda").repeat_interleave(g)
            hidden = torch.arange(keys.shape[0], device="cuda")[None, :] > last[:, None]
            share = torch.softmax(scores.masked_fill(hidden, -math.inf), dim=1)
            out[i, :, head * g:(head + 1) * g] = (share @ values).view(n_q, g, d)
            if gathered is not None:
                gathered[i, head, :lens[i]] += share[:, case["prefix"]:].sum(0)
    return {"out": out, "weights": gathered} if case["weights"] else {"out": out}


def _exact_gemv(case, s):
    y = torch.empty((case["batch"], case["rows"]), dtype=torch.float64, device="cuda")
    x = s["x"].double().t().contiguous()
    for r in range(0, case["rows"], 4096):
        b = s["codes"][r:r + 4096]
        w = torch.empty((b.shape[0], case["cols"]), dtype=torch.float64, device="cuda")
        w[:, ::2], w[:, 1::2] = b.remainder(16).double() - 8, b.div(16, rounding_mode="floor").double() - 8
        w *= s["scales"][r:r + 4096].double().repeat_interleave(case["group"], dim=1)
        if s["bases"] is not None:
            w += s["bases"][r:r + 4096].double().repeat_interleave(case["group"], dim=1)
        y[:, r:r + 4096] = (w @ x).t()
    return y


def _exact_sample(case, s):
    logits = s["logits"].double().cpu().numpy()
    uniforms = s["uniforms"].double().cpu().numpy()
    setting = {name: s[name].double().cpu().numpy() if torch.is_tensor(s[name])
               else np.full(case["rows"], np.float32(s[name]), dtype=np.float64)
               for name in ("temperature", "top_k", "top_p", "min_p")}
    tokens, logprobs = [], []
    for r in range(case["rows"]):
        x = logits[r]
        temperature, k, p, least = (setting[name][r] for name in ("temperature", "top_k", "top_p", "min_p"))
        if temperature <= 0:
            tokens.append(int(np.argmax(x)))
            logprobs.append(0.0)
            continue
        with np.errstate(over="ignore"):
            w = np.exp((x - x.max()) / temperature)
        by_weight = np.lexsort((np.arange(x.size), -x))
        if 0 < k < x.size:
            by_weight = by_weight[:int(k)]
        by_weight = by_weight[w[by_weight] >= LEAST]
        if p < 1:
            sums = np.cumsum(w[by_weight])
            by_weight = by_weight[:int(np.searchsorted(sums, p * sums[-1])) + 1]
        kept = np.sort(by_weight[(w[by_weight] >= least) | (np.arange(by_weight.size) == 0)])
        sums = np.cumsum(w[kept])
        i = min(int(np.searchsorted(sums, uniforms[r] * sums[-1], side="right")), kept.size - 1)
        tokens.append(int(kept[i]))
        logprobs.append(float(np.log(w[kept[i]] / sums[-1])))
    return {"tokens": torch.tensor(tokens, dtype=torch.int32), "logprobs": torch.tensor(logprobs, dtype=torch.float64)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"cache": _exact_cache, "attention": _exact_attention, "gemv": _exact_gemv, "sample": _exact_sample}[
        case["op"]](case, s)
