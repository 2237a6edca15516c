"""Cases of the operators that stand between the compressed products of a decoder layer.

A case is a dict of plain values; `op` names the entry point:

  norm       rms_norm: the residual's addition, the RMS norm and the rounding to what the next product takes
             (or to 8 bits with scales)
  attention  prefix_attention: the new tokens of a batch over one prefix that all sequences share and over each
             sequence's own cache; with `weights`, also the weight that each own key has gathered
  evict      cache_evict: the newest and the heaviest tokens of every sequence moved to a smaller cache

Head counts, head sizes and widths are those of the 7B, 8B and 70B shapes of this repository's workloads
(32 or 64 heads of 128 on 8 or 32 of keys; 4096, 8192 wide; batches of 1 to 16), and generic ones.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1, "none": 0}
EPS = 1e-5
E4M3_MAX = 448.0


def listed():
    return [
        # before a projection in a decode step of one sequence: the product's float32 result joins the residual
        {"name": "norm 1x4096", "op": "norm", "tokens": 1, "hidden": 4096, "x": "f32", "residual": "bf16",
         "out": "bf16", "group": 0},
        # a few prompts packed together, a width that no vector load divides
        {"name": "norm 1021x4100 f16", "op": "norm", "tokens": 1021, "hidden": 4100, "x": "f32", "residual": "f16",
         "out": "f16", "group": 0},
        # a long prompt of the 70B shape, handed on in 8 bits
        {"name": "norm 8192x8192 e4m3", "op": "norm", "tokens": 8192, "hidden": 8192, "x": "bf16",
         "residual": "bf16", "out": "e4m3", "group": 128},
        # one chat at its start, 8B shape: a short system prompt and a few hundred tokens
        {"name": "attn b1 p512", "op": "attention", "type": "bf16", "batch": 1, "queries": 1, "heads": 32,
         "kv_heads": 8, "dim": 128, "prefix": 512, "own": 300, "weights": False},
        # a full decode batch on one long system prompt, 8B shape
        {"name": "attn b16 p8192", "op": "attention", "type": "bf16", "batch": 16, "queries": 1, "heads": 32,
         "kv_heads": 8, "dim": 128, "prefix": 8192, "own": 1024, "weights": False},
        # speculative decoding of three tokens, 7B shape (a key head for each head), odd lengths
        {"name": "attn b5 q3 p1777", "op": "attention", "type": "f16", "batch": 5, "queries": 3, "heads": 32,
         "kv_heads": 32, "dim": 128, "prefix": 1777, "own": 777, "weights": False},
        # a decode batch of the 70B shape that gathers the weights an eviction goes by
        {"name": "attn b8 own4096 weights", "op": "attention", "type": "bf16", "batch": 8, "queries": 1,
         "heads": 64, "kv_heads": 8, "dim": 128, "prefix": 2048, "own": 4096, "weights": True},
        # the sequences' own prompts, a chunk of 256 tokens each, on the shared one
        {"name": "attn b4 q256 p4096", "op": "attention", "type": "bf16", "batch": 4, "queries": 256, "heads": 32,
         "kv_heads": 8, "dim": 128, "prefix": 4096, "own": 512, "weights": False},
        # a batch of questions on one long document, 70B shape
        {"name": "attn b16 p131072", "op": "attention", "type": "bf16", "batch": 16, "queries": 1, "heads": 64,
         "kv_heads": 8, "dim": 128, "prefix": 131072, "own": 2048, "weights": False},
        # one short cache halved
        {"name": "evict b1 1024to512", "op": "evict", "type": "bf16", "batch": 1, "kv_heads": 8, "dim": 128,
         "own": 1024, "keep": 512, "recent": 64},
        # the caches of a decode batch, each of another length (some within the budget already)
        {"name": "evict b16 4096to1000", "op": "evict", "type": "f16", "batch": 16, "kv_heads": 8, "dim": 128,
         "own": 4096, "keep": 1000, "recent": 250},
        # long prompts cut down after their prefill
        {"name": "evict b4 65536to16384", "op": "evict", "type": "bf16", "batch": 4, "kv_heads": 8, "dim": 128,
         "own": 65536, "keep": 16384, "recent": 1024},
    ]


# What a drawn case may cost at most: the largest listed ones.
MOST_NORM = 8192 * 8192
MOST_BYTES = 560 << 20
MOST_SCORES = 128 << 20  # scores of a plain pass


def _log(rng, low, high):
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    op = rng.choice(["norm", "attention", "attention", "evict"])
    if op == "norm":
        out = rng.choice(["f32", "bf16", "f16", "e4m3"])
        hidden = _log(rng, 256, 16384)
        group = rng.choice([0, 32, 64, 128]) if out == "e4m3" else 0
        # widths are multiples of the group, or of 8; now and then they are any number
        step = group or rng.choice([8, 8, 1])
        hidden = hidden // step * step
        return {"op": op, "tokens": _log(rng, 1, min(8192, MOST_NORM // hidden)), "hidden": hidden,
                "x": rng.choice(["f32", "bf16", "f16"]), "residual": rng.choice(["none", "f32", "bf16", "f16"]),
                "out": out, "group": group}
    if op == "evict":
        case = {"op": op, "type": rng.choice(["bf16", "f16"]), "batch": rng.randint(1, 16),
                "kv_heads": rng.choice([1, 4, 8, 32]), "dim": rng.choice([64, 96, 128])}
        case["own"] = _log(rng, 64, 65536)
        while work({**case, "keep": case["own"], "recent": 0})["bytes"] > MOST_BYTES:
            case["own"] = case["own"] // 2 + 1
        case["keep"] = max(1, round(case["own"] * rng.uniform(0.1, 0.9)))
        case["recent"] = round(case["keep"] * rng.uniform(0.0, 0.5))
        return case
    heads, kv_heads = rng.choice([(32, 8), (64, 8), (32, 32), (16, 2), (24, 8)])
    case = {"op": op, "type": rng.choice(["bf16", "f16"]), "batch": rng.randint(1, 16),
            "queries": rng.choice([1, 1, 1, rng.randint(2, 8), _log(rng, 9, 256)]), "heads": heads,
            "kv_heads": kv_heads, "dim": rng.choice([64, 80, 128, 128]), "prefix": _log(rng, 1, 131072),
            "own": 0, "weights": False}
    case["own"] = max(case["queries"], _log(rng, 1, 8192))
    case["weights"] = case["queries"] <= 8 and rng.random() < 0.4
    rows = case["batch"] * case["queries"] * heads
    while rows * (case["prefix"] + case["own"]) > MOST_SCORES or work(case)["bytes"] > MOST_BYTES:
        if case["prefix"] >= case["own"] or case["own"] == case["queries"]:
            case["prefix"] = case["prefix"] // 2 + 1
        else:
            case["own"] = max(case["queries"], case["own"] // 2)
    return case


def _lens(case):
    """Lengths of the sequences' own caches, spread evenly between the least and the capacity."""
    low, high, b = case.get("queries", 1), case["own"], case["batch"]
    return [high - (high - low) * i // b if i else high for i in range(b)]


def _kept(case):
    return [min(n, case["keep"]) for n in _lens(case)]


def work(case):
    if case["op"] == "norm":
        n, t = case["tokens"] * case["hidden"], case["tokens"]
        scales = 0 if case["out"] != "e4m3" else 4 * t * (case["hidden"] // case["group"] if case["group"] else 1)
        each = BYTES[case["x"]] + 2 * BYTES[case["residual"]] + BYTES[case["out"]]
        return {"bytes": n * each + 2 * case["hidden"] + scales, "flops": 5 * n}
    d, h, b = case["dim"], case["kv_heads"], case["batch"]
    if case["op"] == "evict":
        rows = sum(_kept(case)) * h
        scored = sum(n for n in _lens(case) if n > case["keep"]) * h
        return {"bytes": 4 * scored + 4 * d * rows + b * h * case["keep"] * (4 * d + 8) + 8 * b,
                "flops": scored}
    n, q = sum(_lens(case)), case["queries"]
    io = 4 * b * q * case["heads"] * d
    seen = q * (b * case["prefix"] + n) - b * q * (q - 1) // 2
    return {"bytes": 4 * d * h * (case["prefix"] + n) + io + (8 * b * h * case["own"] if case["weights"] else 0),
            "flops": 4 * d * case["heads"] * seen}


def _rand(g, shape, scale=1.0, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def _keys(g, shape, dtype):
    """Keys or values [.., heads, dim]: tokens differ, and each head has channels that stand out in all of them."""
    t = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    t += _rand(g, shape[-2:], 0.5)
    return t.to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if case["op"] == "norm":
        n, t = case["hidden"], case["tokens"]
        # hidden states: a few channels far larger than the rest
        size = 1 + 20 * (torch.rand(n, generator=g, device="cuda") < 0.005).float()
        state = {"x": (_rand(g, (t, n), 0.3) * size).to(TYPE[case["x"]]),
                 "residual": None, "weight": (1 + _rand(g, (n,), 0.1)).to(torch.bfloat16)}
        if case["residual"] != "none":
            state["residual"] = (_rand(g, (t, n)) * size).to(TYPE[case["residual"]])
        return {**state, "case": dict(case)}
    b, h, d, dtype = case["batch"], case["kv_heads"], case["dim"], TYPE[case["type"]]
    order = torch.randperm(b, generator=g, device="cuda")
    state = {"k": _keys(g, (b, case["own"], h, d), dtype), "v": _keys(g, (b, case["own"], h, d), dtype),
             "lens": torch.tensor(_lens(case), dtype=torch.int32, device="cuda")[order].contiguous(),
             "case": dict(case)}
    if case["op"] == "evict" or case["weights"]:
        # gathered weight falls off steeply: a few tokens (some of them equal) hold most, many have next to none
        u = torch.rand((b, h, case["own"]), generator=g, device="cuda").clamp_(min=1e-3)
        state["weights"] = u.pow_(-1.2).mul_(1e-3)
    if case["op"] == "attention":
        state["q"] = _rand(g, (b, case["queries"], case["heads"], d), 2.0, dtype)
        state["prefix_k"] = _keys(g, (case["prefix"], h, d), dtype)
        state["prefix_v"] = _keys(g, (case["prefix"], h, d), dtype)
    return state


def _plain_norm(s):
    case = s["case"]
    t = s["x"].float()
    outs = {}
    if s["residual"] is not None:
        t = t + s["residual"].float()
        outs["sum"] = t.to(s["residual"].dtype)
    y = t * torch.rsqrt((t * t).mean(dim=-1, keepdim=True) + EPS) * s["weight"].float()
    if case["out"] != "e4m3":
        outs["out"] = y.to(TYPE[case["out"]])
        return outs
    groups = y.view(y.shape[0], -1, case["group"] or y.shape[1])
    scale = groups.abs().amax(dim=-1, keepdim=True) / E4M3_MAX
    scale = torch.where(scale > 0, scale, torch.ones_like(scale))
    outs["out"] = (groups / scale).clamp(-E4M3_MAX, E4M3_MAX).view(y.shape).to(torch.float8_e4m3fn)
    outs["scale"] = scale.squeeze(-1)
    return outs


def _plain_attention(s):
    q, k, v, pk, pv = (s[n].float() for n in ("q", "k", "v", "prefix_k", "prefix_v"))
    b, n_q, heads, d = q.shape
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


def _plain_evict(s):
    keep, recent, w = s["case"]["keep"], s["case"]["recent"], s["weights"]
    b, h, cap = w.shape
    n = s["lens"].long()[:, None, None]
    at = torch.arange(cap, device=w.device)
    rank = torch.where(at >= n - recent, torch.full_like(w, math.inf), w)
    rank = torch.where(at >= n, torch.full_like(w, -math.inf), rank)
    slots = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :keep]
    slots = torch.where(slots < n, slots, torch.full_like(slots, cap))
    slots = torch.sort(slots, dim=-1).values
    there = slots < cap
    source = torch.where(there, slots, torch.zeros_like(slots))
    rows = source.permute(0, 2, 1)[..., None].expand(b, keep, h, s["k"].shape[3])
    there_rows = there.permute(0, 2, 1)[..., None]
    k, v = (torch.where(there_rows, torch.gather(t, 1, rows), torch.zeros((), dtype=t.dtype, device=t.device))
            for t in (s["k"], s["v"]))
    weights = torch.where(there, torch.gather(w, 2, source), torch.zeros_like(w[..., :1]))
    return {"k": k, "v": v, "weights": weights, "lens": s["lens"].clamp(max=keep),
            "slots": torch.where(there, slots, torch.full_like(slots, -1)).to(torch.int32)}


def _own_norm(s):
    import paper_2502_00922_amd as hl
    case = s["case"]
    r = hl.rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS, out_dtype=TYPE[case["out"]],
                    group=case["group"])
    return {name: t for name, t in zip(("out", "sum", "scale"), r) if t is not None}


def _own_attention(s):
    import paper_2502_00922_amd as hl
    r = hl.prefix_attention(s["q"], s["k"], s["v"], s["lens"], prefix_k=s["prefix_k"], prefix_v=s["prefix_v"],
                            weights=s["weights"] if s["case"]["weights"] else None)
    return {"out": r[0], "weights": r[1]} if s["case"]["weights"] else {"out": r[0]}


def _own_evict(s):
    import paper_2502_00922_amd as hl
    r = hl.cache_evict(s["k"], s["v"], s["weights"], s["lens"], keep=s["case"]["keep"], recent=s["case"]["recent"])
    return dict(zip(("k", "v", "weights", "lens", "slots"), r))


def run(state):
    op = state["case"]["op"]
    if own:
        return {"norm": _own_norm, "attention": _own_attention, "evict": _own_evict}[op](state)
    return {"norm": _plain_norm, "attention": _plain_attention, "evict": _plain_evict}[op](state)


def _exact_evict(case, s):
    b, h, keep, d = case["batch"], case["kv_heads"], case["keep"], case["dim"]
    k, v = (torch.zeros((b, keep, h, d), dtype=torch.float64, device="cuda") for _ in range(2))
    weights = torch.zeros((b, h, keep), dtype=torch.float64, device="cuda")
    slots = torch.full((b, h, keep), -1, dtype=torch.int32, device="cuda")
    lens, gathered = s["lens"].tolist(), s["weights"].double().cpu().numpy()
    for i in range(b):
        n = lens[i]
        old = max(0, n - case["recent"]) if n > keep else 0
        for head in range(h):
            w = gathered[i, head, :old]
            best = np.lexsort((np.arange(old), -w))[:keep - case["recent"]]
            at = np.concatenate([np.sort(best), np.arange(old, n)])
            at = torch.from_numpy(at.astype(np.int64)).to("cuda")
            m = at.numel()
            k[i, :m, head], v[i, :m, head] = s["k"][i, at, head].double(), s["v"][i, at, head].double()
            weights[i, head, :m] = s["weights"][i, head, at].double()
            slots[i, head, :m] = at.int()
    return {"k": k, "v": v, "weights": weights, "lens": s["lens"].clamp(max=keep), "slots": slots}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        t = s["x"].double()
        outs = {}
        if s["residual"] is not None:
            t = t + s["residual"].double()
            outs["sum"] = t
        y = t / torch.sqrt(torch.mean(t ** 2, -1, keepdim=True) + EPS) * s["weight"].double()
        if case["out"] == "e4m3":
            size = case["group"] or case["hidden"]
            top = y.abs().unflatten(1, (-1, size)).amax(2)
            outs["scale"] = torch.where(top > 0, top / E4M3_MAX, 1.0)
            y = y / outs["scale"].repeat_interleave(size, dim=1)
        outs["out"] = y
        return outs
    if case["op"] == "evict":
        return _exact_evict(case, s)
    b, n_q, heads, d = s["q"].shape
    g = heads // case["kv_heads"]
    out = torch.zeros((b, n_q, heads, d), dtype=torch.float64, device="cuda")
    gathered = s["weights"].double() if case["weights"] else None
    lens = s["lens"].tolist()
    for head in range(case["kv_heads"]):
        for i in range(b):
            keys = torch.cat([s["prefix_k"][:, head], s["k"][i, :lens[i], head]]).double()
            values = torch.cat([s["prefix_v"][:, head], s["v"][i, :lens[i], head]]).double()
            rows = s["q"][i, :, head * g:(head + 1) * g].double().reshape(n_q * g, d)
            scores = rows @ keys.t().contiguous() / math.sqrt(d)
            last = case["prefix"] + lens[i] - n_q + torch.arange(n_q, device="cuda").repeat_interleave(g)
            hidden = torch.arange(keys.shape[0], device="cuda")[None, :] > last[:, None]
            share = torch.softmax(scores.masked_fill(hidden, -math.inf), dim=1)
            out[i, :, head * g:(head + 1) * g] = (share @ values).view(n_q, g, d)
            if gathered is not None:
                gathered[i, head, :lens[i]] += share[:, case["prefix"]:].sum(0)
    return {"out": out, "weights": gathered} if case["weights"] else {"out": out}
