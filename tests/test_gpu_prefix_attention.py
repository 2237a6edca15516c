"""prefix_attention against the definition in 64 bits (MI355X).

Bounds of an output: one rounding to its type (u: 2^-8 for bf16, 2^-11 for float16); p is rounded to the same type
before it meets v (u again, of sum p|v|); a score is a float32 sum of dim products, so it is off by at most
e = (dim + 4) * 2^-24 * max sum |q k| * scale, which moves a weight and the sum under it by at most a factor exp(e)
each; the sums of weights and of parts add at most 64 * 2^-24. float16 weights below 2^-14 are spaced 2^-24: half of
that for each key (the kernel's weights are at least these in their own units, where the sum is 1 or more)."""
import math

import pytest
import torch

import paper_2502_00922_amd as hl

pytestmark = pytest.mark.gpu
U = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}
TYPES = [torch.bfloat16, torch.float16]


def make(dtype, batch, queries, heads, kv_heads, dim, prefix, own, lens=None, size=1.5, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    c = {"q": (size * rand(batch, queries, heads, dim)).to(dtype)}
    if own:
        c["k"], c["v"] = rand(batch, own, kv_heads, dim).to(dtype), rand(batch, own, kv_heads, dim).to(dtype)
        if lens is None:
            lens = [own - (own - min(queries, own)) * i // max(batch, 1) for i in range(batch)]
        c["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if prefix:
        c["prefix_k"], c["prefix_v"] = rand(prefix, kv_heads, dim).to(dtype), rand(prefix, kv_heads, dim).to(dtype)
    return c


def reference(c, scale=None):
    """out, lse, own weights, sum p|v| and the largest sum |q k| * scale, on the CPU in 64 bits."""
    q = c["q"].double().cpu()
    batch, queries, heads, dim = q.shape
    scale = 1 / math.sqrt(dim) if scale is None else scale
    some = c["k"] if "k" in c else c["prefix_k"]
    kv_heads, share = some.shape[-2], heads // some.shape[-2]
    cap = c["k"].shape[1] if "k" in c else 0
    out, size = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full((batch, queries, heads), -math.inf, dtype=torch.float64)
    weights = torch.zeros((batch, kv_heads, cap), dtype=torch.float64)
    none = torch.zeros((0, dim), dtype=torch.float64)
    most = 0.0
    for b in range(batch):
        n = min(max(int(c["lens"][b]), 0), cap) if cap else 0
        for h in range(kv_heads):
            pk, pv = (c[x][:, h].double().cpu() if "prefix_k" in c else none for x in ("prefix_k", "prefix_v"))
            ok, ov = (c[x][b, :n, h].double().cpu() if cap else none for x in ("k", "v"))
            for i in range(queries):
                seen = max(0, n - (queries - 1 - i))
                keys, values = torch.cat([pk, ok[:seen]]), torch.cat([pv, ov[:seen]])
                if not len(keys):
                    continue
                rows = q[b, i, h * share:(h + 1) * share]
                s = rows @ keys.T * scale
                most = max(most, float((rows.abs() @ keys.abs().T).max()) * abs(scale))
                p = torch.softmax(s, 1)
                out[b, i, h * share:(h + 1) * share] = p @ values
                size[b, i, h * share:(h + 1) * share] = p @ values.abs()
                lse[b, i, h * share:(h + 1) * share] = torch.logsumexp(s, 1)
                weights[b, h, :seen] += p[:, len(pk):].sum(0)
    return out, lse, weights, size, most


def check(c, scale=None, **more):
    q = c["q"]
    batch, queries, heads, dim = q.shape
    lse = torch.full((batch, queries, heads), 77.0, device="cuda")
    start = None
    if "k" in c:
        kv_heads, cap = c["k"].shape[2], c["k"].shape[1]
        start = torch.rand((batch, kv_heads, cap), device="cuda")
        more = {**more, "weights": start.clone()}
    r = hl.prefix_attention(**c, scale=scale, lse=lse, **more)
    out, want_lse, weights, size, most = reference(c, scale)
    u = U[q.dtype]
    e = (dim + 4) * 2.0**-24 * most
    keys = (c["k"].shape[1] if "k" in c else 0) + (len(c["prefix_k"]) if "prefix_k" in c else 0)
    v_max = max(float(c[x].float().abs().max()) for x in ("v", "prefix_v") if x in c)
    tiny = keys * 2.0**-25 * v_max if q.dtype == torch.float16 else 0.0
    bound = u * out.abs() + (u + 2 * e + 64 * 2.0**-24) * (1 + u) * size + tiny + 2.0**-25
    got = r.out.double().cpu()
    assert ((got - out).abs() <= bound).all(), float(((got - out).abs() / bound).max())
    empty = want_lse == -math.inf
    assert (got[empty] == 0).all() and (r.lse.double().cpu()[empty] == -math.inf).all()
    d = (r.lse.double().cpu() - want_lse)[~empty].abs()
    assert (d <= e + 64 * 2.0**-24 + 4 * 2.0**-24 * want_lse[~empty].abs()).all()
    if start is not None:
        w = start.double().cpu() + weights
        err = (r.weights.double().cpu() - w).abs()
        assert (err <= (2 * e + 80 * 2.0**-24) * weights + 2.0**-23 * w + 1e-12).all()
    return r


SHAPES = [  # batch, queries, heads, kv_heads, dim, prefix, own
    (1, 1, 1, 1, 64, 0, 1), (1, 1, 1, 1, 64, 1, 0), (1, 1, 4, 4, 8, 5, 3), (2, 1, 4, 2, 40, 31, 33),
    (1, 1, 32, 8, 128, 512, 300), (16, 1, 32, 8, 128, 129, 65), (3, 1, 64, 8, 128, 127, 128), (5, 3, 8, 8, 128, 177, 77),
    (4, 2, 24, 8, 80, 33, 200), (2, 5, 12, 2, 96, 100, 131), (7, 1, 16, 2, 256, 70, 45), (2, 9, 4, 1, 160, 50, 40),
    (5, 9, 16, 4, 128, 300, 64), (2, 40, 8, 2, 128, 90, 111), (3, 33, 8, 1, 64, 65, 33), (70, 1, 4, 2, 64, 40, 19),
    (130, 1, 2, 1, 128, 17, 9), (2, 70, 4, 2, 256, 40, 90), (1, 1, 8, 8, 128, 3001, 0), (1, 1, 8, 8, 128, 0, 3001),
    (2, 7, 6, 3, 24, 260, 7), (1, 200, 4, 1, 128, 0, 200)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(dtype, shape):
    check(make(dtype, *shape))


@pytest.mark.parametrize("queries,lens", [(1, [0, 1, 2, 64, 63, 65]), (4, [0, 1, 2, 3, 4, 5]), (3, [-5, 1000, 96, 31, 32, 33])])
@pytest.mark.parametrize("prefix", [0, 37])
def test_lengths(queries, lens, prefix):
    # among them sequences without a key, and tokens that see none
    check(make(torch.bfloat16, 6, queries, 8, 2, 64, prefix, 96, lens=lens))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [0.0, 10.0, 60.0])
def test_flat_and_steep(dtype, size):
    check(make(dtype, 2, 2, 8, 2, 128, 500, 300, size=size))


@pytest.mark.parametrize("scale", [-0.3, 0.0, 2.0])
def test_scale(scale):
    check(make(torch.float16, 2, 2, 4, 2, 64, 100, 90), scale=scale)


def test_maximum_grows_along_the_keys():
    # every step's scores pass the ones before by more than the slack
    c = make(torch.bfloat16, 2, 1, 8, 2, 128, 900, 600)
    c["q"][...] = 1
    c["prefix_k"][...] = (torch.arange(900, device="cuda") / 300).view(-1, 1, 1)
    c["k"][...] = 3 + (torch.arange(600, device="cuda") / 300).view(1, -1, 1, 1)
    check(c)


def test_strides():
    base = make(torch.bfloat16, 3, 2, 8, 4, 80, 150, 90)
    want = hl.prefix_attention(**base).out
    c = dict(base)
    c["k"] = base["k"].transpose(1, 2).contiguous().transpose(1, 2)      # heads before tokens
    wide = torch.randn(3, 100, 4, 176, device="cuda").to(torch.bfloat16)  # keys and values in one buffer
    wide[:, 5:95, :, 88:168] = base["v"]
    c["v"] = wide[:, 5:95, :, 88:168]
    both = torch.zeros(400, 4, 2, 80, device="cuda", dtype=torch.bfloat16)
    both[100:250, :, 0], both[100:250, :, 1] = base["prefix_k"], base["prefix_v"]
    c["prefix_k"], c["prefix_v"] = both[100:250, :, 0], both[100:250, :, 1]
    assert torch.equal(hl.prefix_attention(**c).out, want)
    check(c)
    c["k"], c["v"] = (base[x][:1].expand(3, -1, -1, -1) for x in ("k", "v"))  # one cache for all
    check(c)


def test_offsets_past_32_bits():
    rows, stride = 70, (1 << 25) - 8
    big = torch.empty(rows * stride + 64, dtype=torch.bfloat16, device="cuda")
    k = big.as_strided((1, rows, 1, 64), (0, stride, 64, 1))
    base = make(torch.bfloat16, 1, 1, 4, 1, 64, 0, rows)
    k.copy_(base["k"])
    want = hl.prefix_attention(**base).out
    assert torch.equal(hl.prefix_attention(base["q"], k, base["v"], base["lens"]).out, want)
    k.copy_(base["v"])
    assert torch.equal(hl.prefix_attention(base["q"], base["k"], k, base["lens"]).out, want)
    got = hl.prefix_attention(base["q"], prefix_k=base["k"][0], prefix_v=k[0]).out
    assert torch.equal(got, hl.prefix_attention(base["q"], prefix_k=base["k"][0], prefix_v=base["v"][0]).out)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_not_there_does_not_count(dtype, bad):
    lens = [0, 5, 63, 64]
    c = make(dtype, 4, 1, 8, 2, 128, 50, 100, lens=lens)
    want = check(c)
    for b, n in enumerate(lens):
        c["k"][b, n:], c["v"][b, n:] = bad, bad
    got = hl.prefix_attention(**c)
    assert torch.equal(got.out, want.out)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_later_tokens_do_not_reach_earlier_ones(dim, bad):
    c = make(torch.bfloat16, 2, 5, 8, 2, dim, 20, 60, lens=[60, 33])
    want = hl.prefix_attention(**c).out.clone()
    for x in ("k", "v"):
        c[x][0, 58], c[x][1, 31] = bad, bad  # the last token but one
    got = hl.prefix_attention(**c).out
    assert torch.equal(got[:, :3], want[:, :3])
    assert not got[:, 3:].isfinite().all(-1).any()
    c["k"][...] = make(torch.bfloat16, 2, 5, 8, 2, dim, 20, 60)["k"]
    got = hl.prefix_attention(**c).out
    assert torch.equal(got[:, :3], want[:, :3])
    if bad == math.inf:  # only the values: each output column is infinite
        assert (got[:, 3:] == math.inf).all()


def test_nan_stays_in_its_row():
    c = make(torch.float16, 3, 1, 8, 2, 128, 400, 100)
    want = hl.prefix_attention(**c).out.clone()
    c["q"][1, 0, 3, 7] = float("nan")
    got = hl.prefix_attention(**c).out
    assert got[1, 0, 3].isnan().all()
    got[1, 0, 3] = want[1, 0, 3]
    assert torch.equal(got, want)


def test_weights_in_place_and_absent():
    c = make(torch.bfloat16, 2, 1, 16, 4, 128, 64, 200)
    zero = hl.prefix_attention(**c, weights_out=torch.empty(2, 4, 200, device="cuda")).weights
    w = torch.rand(2, 4, 200, device="cuda")
    apart = hl.prefix_attention(**c, weights=w).weights
    assert apart is not w and torch.equal(apart, w + zero)
    hl.prefix_attention(**c, weights=w, weights_out=w)
    assert torch.equal(w, apart)
    beyond = torch.arange(200, device="cuda")[None, None] >= c["lens"][:, None, None]
    assert (zero[beyond.expand(2, 4, 200)] == 0).all()


def test_repeats_streams_and_workspace():
    c = make(torch.bfloat16, 9, 1, 32, 8, 128, 2000, 700)
    want = hl.prefix_attention(**c, weights_out=torch.empty(9, 8, 700, device="cuda"))
    for _ in range(3):
        got = hl.prefix_attention(**c, weights_out=torch.empty(9, 8, 700, device="cuda"))
        assert torch.equal(got.out, want.out) and torch.equal(got.weights, want.weights)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = hl.prefix_attention(**c)
    s.synchronize()
    assert torch.equal(got.out, want.out)
    ws = torch.full((1 << 26,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN everywhere
    assert torch.equal(hl.prefix_attention(**c, workspace=ws).out, want.out)


def test_graph_replays_with_other_lengths():
    c = make(torch.bfloat16, 4, 1, 16, 4, 128, 300, 260)
    out, lengths = torch.empty_like(c["q"]), [[260, 1, 100, 0], [7, 130, 260, 129], [260, 260, 260, 260]]
    hl.prefix_attention(**c, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        hl.prefix_attention(**c, out=out)
    for n in lengths + lengths:
        c["lens"].copy_(torch.tensor(n, dtype=torch.int32))
        g.replay()
        got = out.clone()
        torch.cuda.synchronize()
        assert torch.equal(got, hl.prefix_attention(**c).out)


def test_refusals():
    c = make(torch.bfloat16, 2, 1, 8, 2, 64, 40, 30)
    bad = [dict(q=c["q"].float()), dict(q=c["q"].cpu()), dict(q=c["q"][0]), dict(k=c["k"].half()), dict(v=c["v"][:, :20]),
           dict(lens=None), dict(lens=c["lens"].long()), dict(lens=c["lens"][:1]), dict(k=c["k"][:1], v=c["v"][:1]),
           dict(prefix_k=c["prefix_k"][:, :1], prefix_v=c["prefix_v"][:, :1]), dict(prefix_v=None),
           dict(q=c["q"][:, :, :7].contiguous()), dict(out=torch.empty_like(c["q"]).float()),
           dict(weights=torch.empty(2, 2, 29, device="cuda")), dict(lse=torch.empty(2, 8, device="cuda")),
           dict(k=c["k"].transpose(2, 3).contiguous().transpose(2, 3)), dict(workspace=torch.empty(8))]
    for b in bad:
        with pytest.raises(ValueError):
            hl.prefix_attention(**{**c, **b})
    with pytest.raises(ValueError):
        hl.prefix_attention(c["q"])
    with pytest.raises(ValueError):
        hl.prefix_attention(c["q"], prefix_k=c["prefix_k"], prefix_v=c["prefix_v"],
                            weights=torch.empty(2, 2, 30, device="cuda"))
    with pytest.raises(hl.HLError):
        hl.prefix_attention(**c, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    odd = torch.zeros(2, 1, 8, 60, dtype=torch.bfloat16, device="cuda")  # a head that is no multiple of 8
    with pytest.raises(hl.HLError):
        hl.prefix_attention(odd, prefix_k=odd[0], prefix_v=odd[0])
    wide = torch.zeros(2, 1, 8, 264, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(hl.HLError):
        hl.prefix_attention(wide, prefix_k=wide[0], prefix_v=wide[0])
    off = torch.zeros(41 * 2 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(41, 2, 64)  # 8 bytes off
    with pytest.raises(hl.HLError):
        hl.prefix_attention(c["q"], prefix_k=off, prefix_v=off)
