"""prefix_attention4 against the definition in 64 bits on what the rows stand for (MI355X).

Bounds of an output: one rounding to its type (u: 2^-8 for bf16, 2^-11 for float16); w = p * scale and p are rounded to
bf16 (r: 2^-8 of them; for a float16 output to two pieces, 2^-16), and meet code - 8 and base: r of sum p (|scale (code -
8)| + |base|). A score's products are with 16, 64 or 128 + code, less 24, 72 or 136 times q: a group's terms are at most
|q| 279 scale, an instruction adds its 32 products with at most 32 roundings and what it adds them to with one, and the
groups, the bases and the scores' scale take dim / 32 + 6 more. So a score is off by at most e = (39 + dim / 32) * 2^-24 *
max sum |q| (279 scale + |base|) * the scores' scale, which moves a weight and the sum under it, and with them the value
(8 scale + |base| at most), by a factor exp(e) each. The sums of w times 16 or 128 + code, less 24 or 136: those of a step
meet 34 roundings of 279 w and later ones of what is left of them, 8 w at most, two a step of 24 steps a wave at most
(the shapes below) and 8 of waves and parts: (34 * 279 + 56 * 8) w < 96 * 104 w. A base meets 33 + 24 + 8 < 96, and the
sum of p as well.

Calls whose keys meet 256 rows and more in the mean give keys and values back in q's type first: each is off by u of it,
which moves a score by u * sum |q k| and an output by u * sum p |v|, and p itself is rounded to that type (u * sum p |v|;
float16 weights below 2^-14 are spaced 2^-24, half of that for each key)."""
import math

import pytest
import torch

import paper_2502_00922_amd as hl
from rows4 import parts, random_rows, row_bytes

pytestmark = pytest.mark.gpu
U = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}
R = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-16}
TYPES = [torch.bfloat16, torch.float16]


def make(dtype, batch, queries, heads, kv_heads, dim, prefix, own, lens=None, size=1.5, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = {"q": (size * torch.randn((batch, queries, heads, dim), generator=g, device="cuda")).to(dtype)}
    if own:
        c["k"], c["v"] = (random_rows((batch, own, kv_heads), dim, g) for _ in range(2))
        if lens is None:
            lens = [own - (own - min(queries, own)) * i // max(batch, 1) for i in range(batch)]
        c["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if prefix:
        c["prefix_k"], c["prefix_v"] = (random_rows((prefix, kv_heads), dim, g) for _ in range(2))
    return c


def reference(c, scale=None):
    """out, lse, own weights, and of the bounds above: sum p (|scale (code - 8)| + |base|), sum p (104 scale + |base|), e's
    size, sum |p v|, the largest sum |q k| and sum p (8 scale + |base|)."""
    q = c["q"].double().cpu()
    batch, queries, heads, dim = q.shape
    scale = 1 / math.sqrt(dim) if scale is None else scale
    some = c["k"] if "k" in c else c["prefix_k"]
    kv_heads, share = some.shape[-2], heads // some.shape[-2]
    cap = c["k"].shape[1] if "k" in c else 0
    held = {x: parts(c[x], dim) for x in ("k", "v", "prefix_k", "prefix_v") if x in c}
    out, steps, sums, sizes, near = (torch.zeros_like(q) for _ in range(5))
    lse = torch.full((batch, queries, heads), -math.inf, dtype=torch.float64)
    weights = torch.zeros((batch, kv_heads, cap), dtype=torch.float64)
    none = (torch.zeros((0, dim), dtype=torch.float64),) * 3
    most = most_qk = 0.0
    for b in range(batch):
        n = min(max(int(c["lens"][b]), 0), cap) if cap else 0
        for h in range(kv_heads):
            pk, pv = (tuple(t[:, h] for t in held[x]) if x in held else none for x in ("prefix_k", "prefix_v"))
            ok, ov = (tuple(t[b, :n, h] for t in held[x]) if x in held else none for x in ("k", "v"))
            for i in range(queries):
                seen = max(0, n - (queries - 1 - i))
                (kc, ks, kb), (vc, vs, vb) = (tuple(torch.cat([x, y[:seen]]) for x, y in zip(pre, own))
                                              for pre, own in ((pk, ok), (pv, ov)))
                if not len(kc):
                    continue
                at = slice(h * share, (h + 1) * share)
                rows = q[b, i, at]
                s = rows @ (kb + ks * (kc - 8)).T * scale
                most = max(most, float((rows.abs() @ (279 * ks + kb.abs()).T).max()) * abs(scale))
                most_qk = max(most_qk, float((rows.abs() @ (kb + ks * (kc - 8)).abs().T).max()) * abs(scale))
                p = torch.softmax(s, 1)
                sizes[b, i, at] = p @ (vb + vs * (vc - 8)).abs()
                out[b, i, at] = p @ (vb + vs * (vc - 8))
                steps[b, i, at] = p @ ((vs * (vc - 8)).abs() + vb.abs())
                sums[b, i, at] = p @ (104 * vs + vb.abs())
                near[b, i, at] = p @ (8 * vs + vb.abs())
                lse[b, i, at] = torch.logsumexp(s, 1)
                weights[b, h, :seen] += p[:, len(pk[0]):].sum(0)
    return out, lse, weights, steps, sums, most, sizes, most_qk, near


def check(c, scale=None, **more):
    q = c["q"]
    batch, queries, heads, dim = q.shape
    lse = torch.full((batch, queries, heads), 77.0, device="cuda")
    start = None
    if "k" in c:
        start = torch.rand((batch, c["k"].shape[2], c["k"].shape[1]), device="cuda")
        more = {**more, "weights": start.clone()}
    r = hl.prefix_attention4(**c, scale=scale, lse=lse, **more)
    out, want_lse, weights, steps, sums, most, sizes, most_qk, near = reference(c, scale)
    e = (39 + dim // 32) * 2.0**-24 * most
    u = U[q.dtype]
    share = heads // (c["k"] if "k" in c else c["prefix_k"]).shape[-2]
    own, prefix = c["k"].shape[1] if "k" in c else 0, len(c["prefix_k"]) if "prefix_k" in c else 0
    if queries * share * (prefix + own) * batch >= 256 * (prefix + own * batch):
        e += u * most_qk
        keys = own + prefix
        steps = 2 * u / R[q.dtype] * sizes + (keys * 2.0**-25 * sizes.max() / R[q.dtype] if q.dtype == torch.float16 else 0.0)
        near = near + sizes
    bound = u * out.abs() + (1 + u) * (R[q.dtype] * steps + 2 * e * near + 96 * 2.0**-24 * sums) + 2.0**-25
    got = r.out.double().cpu()
    assert ((got - out).abs() <= bound).all(), float(((got - out).abs() / bound).max())
    empty = want_lse == -math.inf
    assert (got[empty] == 0).all() and (r.lse.double().cpu()[empty] == -math.inf).all()
    d = (r.lse.double().cpu() - want_lse)[~empty].abs()
    assert (d <= e + 96 * 2.0**-24 + 4 * 2.0**-24 * want_lse[~empty].abs()).all()
    if start is not None:
        w = start.double().cpu() + weights
        err = (r.weights.double().cpu() - w).abs()
        assert (err <= (2 * e + 96 * 2.0**-24) * weights + 2.0**-23 * w + 1e-12).all()
    return r


SHAPES = [  # batch, queries, heads, kv_heads, dim, prefix, own
    (1, 1, 1, 1, 64, 0, 1), (1, 1, 1, 1, 64, 1, 0), (1, 1, 4, 4, 32, 5, 3), (2, 1, 4, 2, 96, 31, 33),
    (1, 1, 32, 8, 128, 512, 300), (16, 1, 32, 8, 128, 129, 65), (3, 1, 64, 8, 128, 127, 128), (5, 3, 8, 8, 128, 177, 77),
    (4, 2, 24, 8, 160, 33, 200), (2, 5, 12, 2, 96, 100, 131), (7, 1, 16, 2, 256, 70, 45), (2, 9, 4, 1, 192, 50, 40),
    (5, 9, 16, 4, 128, 300, 64), (2, 40, 8, 2, 128, 90, 111), (3, 33, 8, 1, 64, 65, 33), (70, 1, 4, 2, 64, 40, 19),
    (130, 1, 2, 1, 128, 17, 9), (2, 70, 4, 2, 256, 40, 90), (1, 1, 8, 8, 128, 3001, 0), (1, 1, 8, 8, 128, 0, 3001),
    (2, 7, 6, 3, 224, 260, 7), (1, 200, 4, 1, 128, 0, 200), (2, 1, 8, 2, 32, 1500, 700), (3, 2, 6, 2, 96, 1300, 400),
    (2, 1, 8, 4, 160, 1200, 90), (2, 1, 8, 4, 192, 1200, 90), (2, 1, 8, 4, 224, 1200, 90), (2, 1, 8, 4, 256, 1200, 90),
    (3, 180, 3, 1, 64, 77, 200), (16, 16, 8, 2, 96, 130, 50), (2, 300, 2, 1, 256, 0, 350), (1, 600, 2, 2, 32, 50, 600),
    (1, 30, 4, 2, 32, 200, 100), (1, 30, 4, 2, 160, 200, 100), (1, 30, 4, 2, 192, 200, 100), (1, 30, 4, 2, 224, 200, 100),
    (300, 1, 4, 2, 64, 100, 19), (40, 4, 4, 1, 128, 500, 30), (1, 256, 1, 1, 64, 0, 256), (1, 255, 1, 1, 64, 0, 255)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(dtype, shape):
    check(make(dtype, *shape))


@pytest.mark.parametrize("queries,lens", [(1, [0, 1, 2, 64, 63, 65]), (4, [0, 1, 2, 3, 4, 5]), (3, [-5, 1000, 96, 31, 32, 33])])
@pytest.mark.parametrize("prefix", [0, 37])
def test_lengths(queries, lens, prefix):
    # among them sequences without a key, and tokens that see none
    check(make(torch.bfloat16, 6, queries, 8, 2, 64, prefix, 96, lens=lens))


@pytest.mark.parametrize("queries,lens", [(1, [0, 1500, 1, 7]), (6, [3, 1500, 0, 1400]), (20, [3, 1500, 0, 1400])])
def test_lengths_in_parts(queries, lens):
    check(make(torch.float16, 4, queries, 8, 2, 128, 0, 1500, lens=lens))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [0.0, 10.0, 40.0])
def test_flat_and_steep(dtype, size):
    check(make(dtype, 2, 2, 8, 2, 128, 500, 300, size=size))


@pytest.mark.parametrize("scale", [-0.3, 0.0, 2.0])
def test_scale(scale):
    check(make(torch.float16, 2, 2, 4, 2, 64, 100, 90), scale=scale)


def test_maximum_grows_along_the_keys():
    # every step's scores pass the ones before by more than the slack
    c = make(torch.bfloat16, 2, 1, 8, 2, 128, 900, 600)
    c["q"][...] = 1
    for x, first in (("prefix_k", 0), ("k", 900)):
        n = c[x].shape[-3]
        base = ((first + torch.arange(n, device="cuda")) / 300).bfloat16().view(n, 1, 1)
        pairs = c[x][..., 64:80].contiguous().view(torch.bfloat16).unflatten(-1, (4, 2))
        pairs[..., 1] = base
        c[x][..., 64:80] = pairs.flatten(-2).view(torch.uint8)
    check(c)


def test_strides():
    c = make(torch.bfloat16, 3, 2, 8, 2, 128, 300, 150)
    a = check(c)
    by_head = {x: c[x].transpose(-3, -2).contiguous().transpose(-3, -2) for x in ("k", "v", "prefix_k", "prefix_v")}
    wide = torch.zeros((3, 150, 2, 3 * 80), dtype=torch.uint8, device="cuda")
    wide[..., 80:160] = c["v"]
    wide[..., 160:] = 0xFF
    wide[..., :80] = 0xFF
    for other in (by_head, {**by_head, "v": wide[..., 80:160]}):
        b = hl.prefix_attention4(**{**c, **other})
        assert torch.equal(a.out, b.out)


def nan_rows(t):
    t[...] = 0xFF  # codes 15, scales and bases NaN


@pytest.mark.parametrize("queries", [1, 3, 20, 130])
@pytest.mark.parametrize("own", [140, 1300])
@pytest.mark.parametrize("dim", [96, 128, 256])
def test_unseen_rows_may_hold_anything(queries, own, dim):
    lens = [own - 1, own // 2, queries, 0]
    c = make(torch.bfloat16, 4, queries, 8, 2, dim, 40, own, lens=lens)
    clean = check(c)
    for b, n in enumerate(lens):
        nan_rows(c["k"][b, n:]), nan_rows(c["v"][b, n:])
    dirty = hl.prefix_attention4(**c)
    assert torch.equal(clean.out, dirty.out)


@pytest.mark.parametrize("queries", [4, 20, 256])
def test_new_tokens_of_nan_reach_only_those_that_see_them(queries):
    lens = [queries + 50, queries + 44, queries]
    c = make(torch.bfloat16, 3, queries, 4, 2, 128, 30, queries + 50, lens=lens)
    clean = hl.prefix_attention4(**c).out
    for b, n in enumerate(lens):
        nan_rows(c["v"][b, n - 2:n])
    got = hl.prefix_attention4(**c).out
    assert torch.equal(got[:, :-2], clean[:, :-2]) and got[:, -2:].isnan().all()
    for b, n in enumerate(lens):
        nan_rows(c["k"][b, n - 1:n])
    got = hl.prefix_attention4(**c).out
    assert torch.equal(got[:, :-2], clean[:, :-2]) and got[:, -2:].isnan().all()


def test_one_group_of_nan():
    # other columns are as they were
    c = make(torch.float16, 2, 1, 4, 2, 128, 50, 60)
    clean = hl.prefix_attention4(**c).out
    c["prefix_v"][7, 1, 64 + 4:64 + 8] = 0xFF
    got = hl.prefix_attention4(**c).out
    assert got[:, :, 2:, 32:64].isnan().all()
    got[:, :, 2:, 32:64] = clean[:, :, 2:, 32:64]
    assert torch.equal(got, clean)


def test_bytes_past_the_pairs_do_not_matter():
    for dim in (32, 64, 96, 160, 224):
        c = make(torch.bfloat16, 2, 2, 4, 2, dim, 40, 50)
        clean = hl.prefix_attention4(**c).out
        for x in ("k", "v", "prefix_k", "prefix_v"):
            c[x][..., dim // 2 + dim // 8:] = 0xFF
        assert torch.equal(hl.prefix_attention4(**c).out, clean)


def test_repeats_are_equal():
    c = make(torch.bfloat16, 5, 1, 32, 8, 128, 3000, 900)
    a, b = (hl.prefix_attention4(**c) for _ in range(2))
    assert torch.equal(a.out, b.out)


def test_captured():
    # replays go by the lengths then
    c = make(torch.bfloat16, 3, 1, 8, 2, 128, 1000, 500, lens=[0, 1, 2])
    w = torch.zeros((3, 2, 500), device="cuda")
    run = lambda: hl.prefix_attention4(**c, weights=w)  # noqa: E731
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c["lens"] += 70
        held = run()
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        eager = run()
        assert torch.equal(held.out, eager.out) and torch.equal(held.weights, eager.weights)


def test_two_streams_at_once():
    c = [make(torch.bfloat16, 4, 1, 32, 8, 128, 4000, 300, seed=i) for i in range(2)]
    want = [hl.prefix_attention4(**x).out for x in c]
    streams = [torch.cuda.Stream() for _ in c]
    torch.cuda.synchronize()
    for _ in range(10):
        got = [hl.prefix_attention4(**x, stream=s).out for x, s in zip(c, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("queries", [1, 20])
def test_far_tokens(queries):
    # tokens so far apart that offsets pass 32 bits
    stride, tokens, n = 1 << 24, 300, row_bytes(128)
    big = torch.empty(tokens * stride + n, dtype=torch.uint8, device="cuda")
    far = big.as_strided((1, tokens, 1, n), (0, stride, n, 1))
    c = make(torch.bfloat16, 1, queries, 4, 1, 128, 0, tokens)
    want = hl.prefix_attention4(**c).out
    for name in ("k", "v"):
        far.copy_(c[name])
        assert torch.equal(hl.prefix_attention4(**{**c, name: far}).out, want)
        assert torch.equal(hl.prefix_attention4(c["q"], prefix_k=c["k"][0], prefix_v=c["v"][0]).out,
                           hl.prefix_attention4(c["q"], prefix_k=(far if name == "k" else c["k"])[0],
                                                prefix_v=(far if name == "v" else c["v"])[0]).out)


@pytest.mark.parametrize("queries", [1, 20, 300])
@pytest.mark.parametrize("sets", ["prefix", "own", "both"])
def test_no_keys(queries, sets):
    # caches without room, prefixes without keys, alone and beside the other set
    own = torch.empty((2, 0, 2, 48), dtype=torch.uint8, device="cuda")
    empty = {"k": own, "v": own, "lens": torch.zeros(2, dtype=torch.int32, device="cuda")} if sets != "prefix" else {}
    if sets != "own":
        empty.update(prefix_k=own[0], prefix_v=own[0])
    c = make(torch.bfloat16, 2, queries, 8, 2, 64, 0 if sets == "prefix" else 90, 90 if sets == "prefix" else 0)
    lse = torch.zeros((2, queries, 8), device="cuda")
    r = hl.prefix_attention4(c["q"], **empty, lse=lse, out=torch.ones_like(c["q"]))
    assert (r.out == 0).all() and (lse == -math.inf).all()
    assert torch.equal(hl.prefix_attention4(**{**empty, **c}).out, hl.prefix_attention4(**c).out)


def test_many_rows_of_other_strides_and_replays():
    # rows that are first given back in 16 bits, from caches that are views, in a graph
    c = make(torch.float16, 3, 128, 8, 2, 96, 200, 150, lens=[150, 128, 0])
    want = check(c)
    wide = {x: torch.full((*c[x].shape[:-3], c[x].shape[-2], c[x].shape[-3], 128), 0xFF, dtype=torch.uint8, device="cuda")
            for x in ("k", "v", "prefix_k", "prefix_v")}
    views = {x: t.transpose(-3, -2)[..., 16:80] for x, t in wide.items()}
    for x, t in views.items():
        t.copy_(c[x])
    views = {**c, **views}
    assert torch.equal(hl.prefix_attention4(**views).out, want.out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = hl.prefix_attention4(**views)
    for n in (140, 128, 150):
        c["lens"][0] = n
        c["q"].copy_(c["q"].flip(0))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held.out, hl.prefix_attention4(**c).out)
